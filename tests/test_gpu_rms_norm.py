"""Root-mean-square norm by degree with the residual's addition, its output in 8 bits, and its adjoint against oracle/residual_oracle.py (fp64).

Tolerances.  The oracle starts from the sum h as it is stored, which is checked to be the exact sum rounded once.  y is h rho gamma with rho off by at
most one rounding, two products and the rounding to the type: 3 U32 + u of |y|.  Codes: half a step of e4m3 around a value
known to 3 U32.  The adjoint: the term gamma dy takes a rounding, the term along h four (rho and the mean, a product each), their difference one, the product
with rho two: 6 U32 of the sum of their magnitudes, and u of the result.  The gradient of gamma: terms known to 3 roundings, fp32 sums of a few dozen of them, then fp64: 32 U32 of the
sum of their magnitudes."""
import numpy as np
import pytest

from oracle import residual_oracle as R
from tests.residual_util import FLOOR, HALF_STEP, U32, check_codes, padding, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    from paper_2507_03840_amd import binding as B
    return B.Egnn(2, 32, 16, 10.0, 200.0)


def tensor(rng, shape, dtype, scale=1.0, planes=0, shift=0):
    """Normal values on the device; planes > 0: inside rows of that many planes more; shift: so many values behind an aligned address."""
    import torch
    n, dim, c = shape
    whole = torch.zeros(n * (dim + planes) * c + shift, dtype=getattr(torch, dtype), device="cuda")
    t = whole[shift:].view(n, dim + planes, c)[:, :dim]
    t.copy_(torch.from_numpy(rng.standard_normal(shape) * scale).to(t.dtype))
    return t


def check(m, n, lmax, c, dtype, residual=True, planes=0, shift=0, scale=1.0, eps=1e-5, seed=0):
    import torch
    rng = np.random.default_rng([seed, n, lmax, c])
    shape = (n, (lmax + 1) ** 2, c)
    x = tensor(rng, shape, dtype, scale, planes, shift)
    r = tensor(rng, shape, dtype, 0.5 * scale, planes, shift) if residual else None
    dy, dh = tensor(rng, shape, dtype, 1.0, planes, shift), tensor(rng, shape, dtype, 1.0, 0, shift)
    gamma = (1 + 0.3 * rng.standard_normal((lmax + 1, c))).astype(np.float32)
    g = torch.from_numpy(gamma).cuda()
    y, h, q, s = m.egnn_rms_norm(x, g, residual=r, eps=eps, q=None)
    if residual:
        assert torch.equal(h, (x.double() + r.double()).to(h.dtype)) if dtype == "float32" else torch.equal(h, (x.float() + r.float()).to(h.dtype))
    else:
        assert h is x
    h64, u, f = values(h), HALF_STEP[dtype], FLOOR[dtype]
    ry = R.rms_norm(h64, gamma, eps)
    assert (np.abs(values(y) - ry) <= (3 * U32 + u) * np.abs(ry) + f).all()
    check_codes(q, s, ry.reshape(-1, c), 3 * U32)
    assert not padding(q).any()
    alone = m.egnn_rms_norm(x, g, residual=r, eps=eps, y=False, h=False, q=None)
    assert alone[0] is None and torch.equal(alone[2].float(), q.float()) and torch.equal(alone[3].view(torch.uint8), s.view(torch.uint8))
    assert torch.equal(m.egnn_rms_norm(x, g, residual=r, eps=eps)[0], y)
    for up in (None, dh):
        dx, dgamma = m.egnn_rms_norm_backward(h, dy, g, dh=up, eps=eps)
        rdx, rdg, size, terms = R.rms_norm_backward(h64, values(dy), gamma, None if up is None else values(up), eps)
        assert (np.abs(values(dx) - rdx) <= 6 * U32 * size + u * np.abs(rdx) + f).all()
        assert (np.abs(values(dgamma) - rdg) <= 32 * U32 * terms + 1e-37).all()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("lmax,c", [(0, 1), (0, 7), (0, 8), (0, 64), (0, 100), (0, 128), (0, 129), (0, 200), (0, 256), (0, 1000), (0, 1001), (1, 1), (1, 33),
                                    (2, 16), (2, 128), (3, 100), (3, 300), (4, 8), (4, 32), (4, 64), (4, 136), (5, 16), (15, 4)])
def test_degrees_and_channels(m, lmax, c, dtype):
    for n in (1, 5, 77):
        check(m, n, lmax, c, dtype, residual=n != 5)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("c", [512, 1024, 2048, 2056, 4096, 4100, 5000, 8192, 20000, 65536])
def test_wide_rows(m, c, dtype):
    for n in (1, 3, 21):
        check(m, n, 0, c, dtype, residual=n != 3)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 1023, 4097, 9001])
def test_lengths(m, n, dtype):
    check(m, n, 0, 32, dtype)
    if n < 2000:
        check(m, n, 4, 16, dtype)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("planes,shift", [(3, 0), (0, 1), (2, 4), (1, 2)])
def test_strides_and_alignment(m, planes, shift, dtype):
    check(m, 50, 2, 32, dtype, planes=planes, shift=shift)
    check(m, 50, 0, 256, dtype, planes=planes, shift=shift)
    check(m, 10, 0, 2048, dtype, planes=planes, shift=shift)


@pytest.mark.parametrize("scale", [1e-30, 1e-8, 1e8, 1e25, 2e37])
def test_magnitudes(m, scale):
    """Squares that fp32 does not hold, and rows far below eps."""
    check(m, 33, 0, 64, "float32", scale=scale, seed=1)
    check(m, 9, 2, 16, "float32", scale=scale, seed=2, eps=1e-12)


def test_rows_of_zeros_and_of_what_is_not_finite(m):
    import torch
    x = torch.randn(9, 4, 40, device="cuda")
    x[1], x[2, 0, 3], x[3, 2, 7], x[4, 1, 0], x[5, 0] = 0.0, float("inf"), float("nan"), -float("inf"), 0.0
    g = torch.ones(2, 40, device="cuda")
    y, _, q, s = m.egnn_rms_norm(x, g, q=None)
    want, bad = R.rms_norm(values(x), np.ones((2, 40))), ~torch.isfinite(x)
    assert torch.isnan(y[2, 0, 3]) and torch.isnan(y[4, 1, 0]) and torch.isnan(y[3, 1:]).all()
    assert (y[2, 0][~bad[2, 0]] == 0).all() and (y[4, 1:][~bad[4, 1:]] == 0).all() and (y[1] == 0).all() and (y[5, 0] == 0).all()
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(values(y))) and np.allclose(values(y)[fine], want[fine], rtol=1e-6)
    v = q.float()
    assert torch.equal(torch.isnan(v), torch.isnan(y)) and (s.view(torch.uint8)[1] == 0).all() and (v[1] == 0).all()
    rows = [0, 6, 7, 8]
    check_codes(q[rows].contiguous(), s[rows].contiguous(), want[rows].reshape(-1, 40), 3 * U32)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lmax,c", [(0, 64), (2, 16), (0, 50), (0, 3000), (5, 8), (0, 30000)])
def test_in_place(m, lmax, c, dtype):
    import torch
    rng = np.random.default_rng(c)
    shape = (40, (lmax + 1) ** 2, c)
    x, r, dy, dh = (tensor(rng, shape, dtype) for _ in range(4))
    g = torch.ones(lmax + 1, c, device="cuda") * 1.5
    y, h, q, s = m.egnn_rms_norm(x, g, residual=r, q=None)
    for into in ("x", "r"):
        a, b = x.clone(), r.clone()
        y2, h2, q2, s2 = m.egnn_rms_norm(a, g, residual=b, h=a if into == "x" else b, q=None)
        assert torch.equal(h2, h) and torch.equal(y2, y) and torch.equal(q2.float(), q.float()) and h2 is (a if into == "x" else b)
        a, b = x.clone(), r.clone()
        y2, h2, q2, _ = m.egnn_rms_norm(a, g, residual=b, y=a if into == "x" else b, q=None)
        assert torch.equal(y2, y) and torch.equal(h2, h) and torch.equal(q2.float(), q.float())
        a, b = x.clone(), r.clone()
        assert torch.equal(m.egnn_rms_norm(a, g, residual=b, y=a if into == "x" else b, h=False)[0], y)
        a, b = x.clone(), r.clone()
        y2, h2, _, _ = m.egnn_rms_norm(a, g, residual=b, h=a if into == "x" else b, y=b if into == "x" else a)
        assert torch.equal(y2, y) and torch.equal(h2, h)
    z = h.clone()
    assert torch.equal(m.egnn_rms_norm(z, g, y=z)[0], y)
    dx, dg = m.egnn_rms_norm_backward(h, dy, g, dh=dh)
    for k in range(3):
        a = [h.clone(), dy.clone(), dh.clone()]
        dx2, dg2 = m.egnn_rms_norm_backward(a[0], a[1], g, dh=a[2], dx=a[k])
        assert torch.equal(dx2, dx) and torch.equal(dg2, dg)
    a = h.clone()
    assert torch.equal(m.egnn_rms_norm_backward(a, dy, g, dh=a)[0], m.egnn_rms_norm_backward(h, dy, g, dh=h.clone())[0])


def test_nothing_beside_the_outputs_is_written(m):
    import torch
    n, c = 37, 20
    x = torch.randn(n, 4, c, device="cuda")
    g = torch.ones(2, c, device="cuda")
    big = torch.full((n, 6, c), 7.0, device="cuda")
    room = torch.full((n * 4, 64), 9, dtype=torch.uint8, device="cuda")
    q = room.view(torch.float8_e4m3fn).view(n, 4, 64)[:, :, :c]
    s = torch.full((n * 4 + 2, 1), 9, dtype=torch.uint8, device="cuda")
    m.egnn_rms_norm(x, g, residual=x, h=big[:, :4], y=False, q=q, scale=s[:n * 4].view(torch.float8_e8m0fnu).view(n, 4, 1))
    assert (big[:, 4:] == 7).all() and (room[:, 32:] == 9).all() and (room[:, 20:32] == 0).all() and (s[n * 4:] == 9).all()
    dx = torch.full((n, 5, c), 7.0, device="cuda")
    m.egnn_rms_norm_backward(x, x, g, dx=dx[:, :4])
    assert (dx[:, 4:] == 7).all() and torch.isfinite(dx).all()


def test_no_rows(m):
    import torch
    g = torch.ones(2, 8, device="cuda")
    x = torch.empty(0, 4, 8, device="cuda")
    y, h, q, s = m.egnn_rms_norm(x, g, residual=x, q=None)
    assert y.shape == (0, 4, 8) and q.shape == (0, 4, 8)
    dx, dg = m.egnn_rms_norm_backward(x, x, g, dgamma=torch.full((2, 8), 5.0, device="cuda"))
    assert (dg == 0).all()


def test_offsets_past_32_bits(m):
    """Rows 100,000 values apart: the last lie behind 2^32 values (8 GB)."""
    import torch
    rng = np.random.default_rng(5)
    n, c = 50000, 64
    x, r, dy = (tensor(rng, (n, 1, c), "float16") for _ in range(3))
    whole = torch.empty((n, 100000), dtype=torch.float16, device="cuda")
    X, S, D, H, Y, G = (whole[:, 1000 * k:1000 * k + c].unsqueeze(1) for k in range(6))
    X.copy_(x), S.copy_(r), D.copy_(dy)
    g = torch.ones(1, c, device="cuda")
    y, h, q, s = m.egnn_rms_norm(x, g, residual=r, q=None)
    dx, dg = m.egnn_rms_norm_backward(h, dy, g)
    _, _, q2, s2 = m.egnn_rms_norm(X, g, residual=S, h=H, y=Y, q=None)
    _, dg2 = m.egnn_rms_norm_backward(H, D, g, dx=G)
    assert torch.equal(H, h) and torch.equal(Y, y) and torch.equal(q2.float(), q.float()) and torch.equal(s2.float(), s.float())
    assert torch.equal(G, dx) and torch.equal(dg2, dg) and torch.equal(X, x) and torch.equal(S, r)


def test_many_rows(m):
    """The gradient of gamma over more rows than workgroups take one by one, all terms of one sign."""
    import torch
    n, c = 200001, 16
    h = torch.rand(n, 1, c, device="cuda") + 1
    dy = torch.rand(n, 1, c, device="cuda") + 1
    g = torch.ones(1, c, device="cuda")
    _, dg = m.egnn_rms_norm_backward(h, dy, g)
    _, want, _, _ = R.rms_norm_backward(values(h), values(dy), np.ones((1, c)))
    assert np.abs(values(dg) / want - 1).max() <= 32 * U32
    for lmax, c in ((5, 3), (4, 7), (1, 300)):
        h, dy = (torch.rand(20001, (lmax + 1) ** 2, c, device="cuda") + 1 for _ in range(2))
        _, dg = m.egnn_rms_norm_backward(h, dy, torch.ones(lmax + 1, c, device="cuda"))
        _, want, _, _ = R.rms_norm_backward(values(h), values(dy), np.ones((lmax + 1, c)))
        assert np.abs(values(dg) / want - 1).max() <= 32 * U32


def test_gradient_against_differences(m):
    """The loss sum(w y) + sum(v h) at moved inputs, evaluated in fp64 from the formulas."""
    import torch
    rng = np.random.default_rng(7)
    shape = (6, 9, 24)
    x, r, w, v = (tensor(rng, shape, "float32") for _ in range(4))
    gamma = (1 + 0.2 * rng.standard_normal((3, 24))).astype(np.float32)
    g = torch.from_numpy(gamma).cuda()
    _, h, _, _ = m.egnn_rms_norm(x, g, residual=r)
    dx, dg = m.egnn_rms_norm_backward(h, w, g, dh=v)
    h64, w64, v64 = values(h), values(w), values(v)
    for _ in range(4):
        a, b, t = rng.standard_normal(shape), rng.standard_normal(gamma.shape), 1e-4
        f = lambda s: (R.rms_norm(h64 + s * a, gamma + s * b) * w64 + (h64 + s * a) * v64).sum()
        want = (f(t) - f(-t)) / (2 * t)
        assert abs((values(dx) * a).sum() + (values(dg) * b).sum() - want) <= 1e-5 * np.abs(values(dx) * a).sum()


def test_captured_and_on_another_stream(m):
    """Replays with eager work between them, two graphs that share a workspace one after the other."""
    import torch
    rng = np.random.default_rng(9)
    shape = (300, 4, 32)
    x, r, dy = (tensor(rng, shape, "float32") for _ in range(3))
    g = torch.ones(2, 32, device="cuda")
    ws = torch.empty(max(256, m.egnn_rms_norm_workspace_bytes(300, 1, 32)), dtype=torch.uint8, device="cuda")
    graphs = []
    stream = torch.cuda.Stream()
    for k in range(2):
        y, h, q, s = m.egnn_rms_norm(x, g, residual=r, q=None)
        dx, dg = m.egnn_rms_norm_backward(h, dy, g, ws=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            m.egnn_rms_norm(x, g, residual=r, y=y, h=h, q=q, scale=s)
            m.egnn_rms_norm_backward(h, dy, g, dx=dx, dgamma=dg, ws=ws)
        graphs.append((graph, y, h, q, s, dx, dg))
    for rep in range(3):
        x.mul_(1.1), dy.mul_(0.9)
        want = m.egnn_rms_norm(x, g, residual=r, q=None)
        back = m.egnn_rms_norm_backward(want[1], dy, g)
        for graph, y, h, q, s, dx, dg in graphs:
            dx.zero_(), y.zero_(), dg.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want[0]) and torch.equal(h, want[1]) and torch.equal(q.float(), want[2].float())
            assert torch.equal(dx, back[0]) and torch.equal(dg, back[1])
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other = m.egnn_rms_norm(x, g, residual=r, q=None)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(other[0], want[0]) and torch.equal(other[2].float(), want[2].float())


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("lmax,c", [(0, 9), (0, 33), (0, 50), (0, 70), (0, 300), (0, 1001), (0, 5003), (1, 33), (2, 50), (4, 13), (1, 601), (5, 7)])
def test_padding_of_rows_that_are_not_finite(m, lmax, c, dtype):
    """The bytes from the last code to the next multiple of 16 are zero whatever the row holds."""
    import torch
    dim = (lmax + 1) ** 2
    x = torch.randn(6, dim, c, device="cuda").to(getattr(torch, dtype))
    x[1, dim - 1, c // 2], x[2, 0, c - 1], x[3, dim - 1, 0], x[4] = float("nan"), float("inf"), -float("inf"), float("nan")
    q = torch.full((6, dim, (c + 15) // 16 * 16), 9, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[..., :c]
    s = torch.full((6, dim, -(-c // 128)), 9, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    y, _, q, s = m.egnn_rms_norm(x, torch.ones(lmax + 1, c, device="cuda"), q=q, scale=s)
    assert not padding(q).any()
    assert torch.equal(torch.isnan(q.float()), torch.isnan(y)) and torch.isnan(y[4]).all() and torch.isnan(y[1, dim - 1]).all()


@pytest.mark.parametrize("c", [4, 5, 8, 12, 32])
def test_terms_that_cancel_in_short_rows(m, c):
    """One value v far above the others, zeros: of gamma dy - h rho^2 <gamma dy h> all but c eps / (v^2 + c eps) cancels, and rho d eps / mean is left.  That
    share is 4.4e-8 at least; in fp64 a dozen roundings of 2^-53 leave it known to 12 * 2^-53 / 4.4e-8 < U32 / 2, gamma = 1 adds none, and the result is
    rounded once: 2 U32."""
    import torch
    rng = np.random.default_rng(c)
    n = 5000
    v, d, at = rng.uniform(15, 30, n).astype(np.float32), rng.uniform(0.5, 2, n).astype(np.float32), rng.integers(0, c, n)
    h, dy = np.zeros((2, n, 1, c), np.float32)
    h[np.arange(n), 0, at], dy[np.arange(n), 0, at] = v, d
    dx, _ = m.egnn_rms_norm_backward(torch.from_numpy(h).cuda(), torch.from_numpy(dy).cuda(), torch.ones(1, c, device="cuda"), eps=1e-5)
    eps = float(np.float32(1e-5))
    mean = v.astype(np.float64) ** 2 / c + eps
    want = d * eps / mean / np.sqrt(mean)
    got = values(dx)[np.arange(n), 0, at]
    assert np.abs(got / want - 1).max() <= 2 * U32


def check_adjoint(m, n, lmax, c, dtype, up=True):
    """The adjoint alone, over more rows than the chunks are."""
    import torch
    rng = np.random.default_rng([3, n, c])
    shape = (n, (lmax + 1) ** 2, c)
    h, dy, dh = (tensor(rng, shape, dtype) for _ in range(3))
    gamma = (1 + 0.3 * rng.standard_normal((lmax + 1, c))).astype(np.float32)
    dx, dgamma = m.egnn_rms_norm_backward(h, dy, torch.from_numpy(gamma).cuda(), dh=dh if up else None)
    rdx, rdg, size, terms = R.rms_norm_backward(values(h), values(dy), gamma, values(dh) if up else None)
    assert (np.abs(values(dx) - rdx) <= 6 * U32 * size + HALF_STEP[dtype] * np.abs(rdx) + FLOOR[dtype]).all()
    assert (np.abs(values(dgamma) - rdg) <= 32 * U32 * terms + 1e-37).all()


@pytest.mark.parametrize("dtype,n,c", [("float32", 2500, 1024), ("float32", 2051, 2044), ("float32", 1100, 4096), ("float32", 1030, 8188), ("float32", 1027, 4097),
                                       ("bfloat16", 2500, 2048), ("bfloat16", 1100, 4096), ("float16", 1030, 8190), ("bfloat16", 2051, 1030),
                                       ("float32", 9001, 300), ("float32", 4099, 512), ("bfloat16", 9001, 1000), ("float16", 8200, 777), ("float32", 1500, 9000)])
def test_adjoint_of_chunks_of_wide_rows(m, dtype, n, c):
    """More rows than chunks (1,024), so that a workgroup's turns follow one another in the same LDS."""
    check_adjoint(m, n, 0, c, dtype, up=n % 2 == 0)


@pytest.mark.parametrize("dtype,n,lmax,c", [("float32", 9001, 1, 64), ("bfloat16", 5003, 4, 40), ("float16", 5000, 2, 300), ("float32", 3001, 3, 33), ("bfloat16", 2501, 5, 16)])
def test_adjoint_of_chunks_of_degrees(m, dtype, n, lmax, c):
    check_adjoint(m, n, lmax, c, dtype)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("lmax,c", [(0, 3), (0, 8), (0, 33), (0, 64), (0, 600), (0, 3000), (1, 16), (2, 50), (4, 8), (5, 3)])
def test_adjoint_of_what_is_not_finite(m, lmax, c, dtype):
    """It stays in its row and degree, and in the channels of gamma whose terms it is in; everything else has the bits that it has without it."""
    import torch
    rng = np.random.default_rng(17)
    shape, l = (40, (lmax + 1) ** 2, c), lmax
    h, dy, dh = (tensor(rng, shape, dtype) for _ in range(3))
    g = torch.from_numpy((1 + 0.3 * rng.standard_normal((lmax + 1, c))).astype(np.float32)).cuda()
    clean, _ = m.egnn_rms_norm_backward(h, dy, g, dh=dh)
    planes = slice(l * l, (l + 1) ** 2)
    h[3, l * l, 1], h[11, l * l, c - 1], h[21, l * l, 0] = float("inf"), float("nan"), -float("inf")
    dy[30, l * l, 2], dh[33, l * l, 1] = float("nan"), float("nan")
    dx, dgamma = m.egnn_rms_norm_backward(h, dy, g, dh=dh)
    bad = torch.zeros(shape, dtype=torch.bool, device="cuda")
    for r in (3, 11, 21, 30):
        bad[r, planes] = True
    bad[33, l * l, 1] = True
    assert torch.isnan(dx[bad]).all() and torch.equal(dx[~bad], clean[~bad])
    assert torch.isnan(dgamma[l]).all() and torch.isfinite(dgamma[:l]).all()             # (a row with a NaN has none but NaN in its norm)
    h[11, l * l, c - 1] = 0.5
    _, dgamma = m.egnn_rms_norm_backward(h, dy, g, dh=dh)
    where = torch.zeros(c, dtype=torch.bool, device="cuda")
    where[:3] = True
    assert torch.isnan(dgamma[l][where]).all() and torch.isfinite(dgamma[l][~where]).all()
