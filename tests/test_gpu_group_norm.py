"""Group norm with SiLU and its adjoint against oracle/block_oracle.py (fp64).

Tolerances.  An output of type t is off by half a step of its own rounding, u_t |value|, and by the fp32 arithmetic before it: xhat is
a difference of values up to max|x| scaled by rstd, so it is off by 4 roundings of (|x| + |mean|) rstd; z, the sigmoid and the product add
about 12 more of max(1, |gamma xhat| + |beta|), and d(SiLU)/dz <= 1.1.  A sum over rows is off by 32 roundings of its
absolute terms (fp32 sums inside a thread of at most a few dozen rows, then fp64) and by what each term dz = dy SiLU'(z), |SiLU'| <= 1.1,
|SiLU''| <= 0.5, is off: SiLU' passes through zero, so that is a part of |dy|, not of |dz|."""
import numpy as np
import pytest

from oracle import block_oracle as K

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
FLOOR = {"float32": 0.0, "float16": 2.0 ** -25, "bfloat16": 0.0}   # half a step of the smallest fp16 numbers


@pytest.fixture(scope="module")
def m():
    from paper_2507_03840_amd import binding as B
    return B.Egnn(2, 32, 16, 10.0, 200.0)


def tensors(rng, n, c, dtype, planes=1, offset=0.5, scale=1.5):
    """A plane of [n][planes][c] on the device, and its values in fp64."""
    import torch
    x = torch.from_numpy(rng.standard_normal((n, planes, c)) * scale + offset).to(getattr(torch, dtype)).cuda()[:, planes // 2]
    return x, x.double().cpu().numpy()


def check(m, n, c, groups, dtype, ptr, planes=1, offset=0.5, scale=1.5, seed=0):
    import torch
    rng = np.random.default_rng([seed, n, c, groups])
    x, x64 = tensors(rng, n, c, dtype, planes, offset, scale)
    dy, dy64 = tensors(rng, n, c, dtype, planes, 0.0, 1.0)
    gamma, beta = (1 + 0.3 * rng.standard_normal(c)).astype(np.float32), (0.3 * rng.standard_normal(c)).astype(np.float32)
    g, b = torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
    p = None if ptr is None else torch.tensor(ptr, dtype=torch.int32, device="cuda")
    y, mean, rstd = m.egnn_group_norm(x, groups, g, b, ptr=p)
    dx, dgamma, dbeta = m.egnn_group_norm_backward(x, dy, mean, rstd, groups, g, b, ptr=p)
    ry, rmean, rrstd = K.group_norm(x64, groups, gamma, beta, ptr)
    rdx, rdg, rdb, sg, sb = K.group_norm_backward(x64, dy64, groups, gamma, beta, ptr)
    at = lambda t: t.double().cpu().numpy()
    big = np.abs(x64).max(initial=0) * 2
    spread = rrstd.max(initial=0)
    z = 4 * U32 * big * spread + 12 * U32 * (1 + np.abs(gamma).max() * big * spread + np.abs(beta).max())
    assert np.abs(at(mean) - rmean).max() <= 2 * U32 * big + U32
    assert np.abs(at(rstd) - rrstd).max() <= 4 * U32 * (1 + big * spread * 2.0 ** -20) * spread
    u, f = HALF_STEP[dtype], FLOOR[dtype]
    rows = ~np.isnan(ry).all(1)
    assert (np.abs(at(y) - ry) <= u * np.abs(ry) + f + 1.1 * z * 1.5)[rows].all()
    # dx: dz is off by 2 z |dy|, the means of dz and of dz xhat by no more, times rstd
    hat = big * spread
    assert (np.abs(at(dx) - rdx) <= u * np.abs(rdx) + f + 8 * z * (1 + hat) * spread * (1 + np.abs(dy64).max(initial=0)) * 1.5)[rows].all()
    assert (np.abs(at(dgamma) - rdg) <= (32 * 1.1 * U32 + 1.5 * z) * sg + 1.5 * 1.1 * z * sb + 1e-30).all()
    assert (np.abs(at(dbeta) - rdb) <= (32 * 1.1 * U32 + 1.5 * z) * sb + 1e-30).all()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("c,groups", [(8, 1), (12, 4), (16, 4), (7, 7), (32, 4), (33, 3), (64, 64), (200, 8), (256, 1), (1001, 7), (1024, 32)])
def test_channels_and_groups(m, c, groups, dtype):
    for n in (1, 5, 333):
        check(m, n, c, groups, dtype, None)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 4095, 20001])
def test_lengths(m, n, dtype):
    check(m, n, 32, 4, dtype, None)


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("ptr", [[0, 0, 1, 1, 3, 50, 50], [0, 1000, 1000, 3001, 3002, 9000], [0, 9000, 9000], [0, 0, 0, 9000],
                                 list(range(0, 901, 3)), [0, 2048, 4096, 6144, 8192]])
def test_ragged_and_empty_segments(m, ptr, dtype):
    check(m, ptr[-1], 64, 8, dtype, ptr)
    check(m, ptr[-1], 16, 4, dtype, ptr, planes=9)


def test_segments_that_span_many_chunks(m):
    check(m, 200000, 32, 4, "float32", [0, 7, 99999, 100000, 200000])
    check(m, 300001, 64, 8, "bfloat16", None, seed=1)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("ptr", [[0] * 20 + [3] * 20 + [5], [0, 4] + [7] * 60 + [900], list(range(0, 1201, 60)), list(range(0, 41))])
def test_many_short_segments(m, ptr, dtype):
    """More segments than rows, one long segment behind many empty ones, a row to a segment."""
    check(m, ptr[-1], 32, 4, dtype, ptr)
    check(m, ptr[-1], 20, 20, dtype, ptr, planes=2)


@pytest.mark.parametrize("dtype", ["float32", "float16"])
def test_a_plane_of_a_node_tensor(m, dtype):
    """x, dy and every output inside [n][25][64]; the rest of the tensors is left alone."""
    import torch
    rng = np.random.default_rng(3)
    n, c, t = 700, 64, getattr(torch, dtype)
    x, x64 = tensors(rng, n, c, dtype, planes=25)
    whole = torch.full((n, 25, c), 5.0, dtype=t, device="cuda")
    one, zero = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    y, mean, rstd = m.egnn_group_norm(x, 8, one, zero, y=whole[:, 0])
    ry, _, _ = K.group_norm(x64, 8, np.ones(c), np.zeros(c))
    assert y.data_ptr() == whole.data_ptr()
    assert np.abs(whole[:, 0].double().cpu().numpy() - ry).max() < 2 * HALF_STEP[dtype] * 8 + 1e-5
    assert (whole[:, 1:] == 5.0).all()
    grad = torch.full((n, 25, c), 5.0, dtype=t, device="cuda")
    m.egnn_group_norm_backward(x, y, mean, rstd, 8, one, zero, dx=grad[:, 3])
    assert (grad[:, :3] == 5.0).all() and (grad[:, 4:] == 5.0).all() and torch.isfinite(grad).all()


def test_offsets_past_32_bits(m):
    """Rows 100,000 values apart: the last lie behind 2^32 values (8 GB)."""
    import torch
    rng = np.random.default_rng(5)
    n, c = 50000, 64
    x, _ = tensors(rng, n, c, "float16")
    dy, _ = tensors(rng, n, c, "float16", 1, 0.0, 1.0)
    whole = torch.empty((n, 100000), dtype=torch.float16, device="cuda")
    X, D, Y, G = (whole[:, 1000 * k:1000 * k + c] for k in range(4))
    X.copy_(x), D.copy_(dy)
    one, zero = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    y, mean, rstd = m.egnn_group_norm(x, 8, one, zero)
    dx, dg, db = m.egnn_group_norm_backward(x, dy, mean, rstd, 8, one, zero)
    _, mean2, rstd2 = m.egnn_group_norm(X, 8, one, zero, y=Y)
    _, dg2, db2 = m.egnn_group_norm_backward(X, D, mean, rstd, 8, one, zero, dx=G)
    assert torch.equal(X, x) and torch.equal(D, dy)
    assert torch.equal(Y, y) and torch.equal(mean2, mean) and torch.equal(rstd2, rstd)
    assert torch.equal(G, dx) and torch.equal(dg2, dg) and torch.equal(db2, db)


def test_in_place(m):
    import torch
    rng = np.random.default_rng(4)
    x, _ = tensors(rng, 5000, 64, "float32")
    x = x.contiguous()
    one, zero = torch.ones(64, device="cuda"), torch.zeros(64, device="cuda")
    y, mean, rstd = m.egnn_group_norm(x, 8, one, zero)
    z = x.clone()
    m.egnn_group_norm(z, 8, one, zero, y=z)
    assert torch.equal(y, z)
    dy = torch.randn_like(x)
    dx, _, _ = m.egnn_group_norm_backward(x, dy, mean, rstd, 8, one, zero)
    m.egnn_group_norm_backward(x, dy, mean, rstd, 8, one, zero, dx=dy)
    assert torch.equal(dx, dy)


def test_large_mean_and_outlier(m):
    """The variance is that about the mean: rows near 1,000 with a spread of 0.01, and one row far from all others."""
    check(m, 3000, 32, 4, "float32", None, offset=1000.0, scale=0.01)
    import torch
    rng = np.random.default_rng(5)
    x = rng.standard_normal((3000, 32)).astype(np.float32)
    x[0] = 1e4
    one, zero = torch.ones(32, device="cuda"), torch.zeros(32, device="cuda")
    _, mean, rstd = m.egnn_group_norm(torch.from_numpy(x).cuda(), 4, one, zero)
    _, rmean, rrstd = K.group_norm(x, 4, np.ones(32), np.zeros(32))
    assert np.abs(mean.cpu().numpy() / rmean - 1).max() < 4 * U32
    assert np.abs(rstd.cpu().numpy() / rrstd - 1).max() < 4 * U32


def test_constant_rows_and_far_values(m):
    """Zero variance: rstd = 1 / sqrt(eps), y = SiLU(beta).  Large |z|: SiLU goes to z and to 0 without NaN."""
    import torch
    x = torch.full((100, 16), 3.0, device="cuda")
    beta = torch.linspace(-200, 200, 16, device="cuda")
    y, mean, rstd = m.egnn_group_norm(x, 4, torch.ones(16, device="cuda"), beta)
    assert torch.equal(mean, torch.full_like(mean, 3.0)) and (rstd * 1e-5 ** 0.5 - 1).abs().max() < 1e-6
    want = beta.double() * torch.sigmoid(beta.double())
    assert (y.double() - want).abs().max() <= 200 * 4 * U32 * 100
    dx, dgamma, dbeta = m.egnn_group_norm_backward(x, torch.ones_like(x), mean, rstd, 4, torch.ones(16, device="cuda"), beta)
    assert torch.isfinite(dx).all() and torch.isfinite(dgamma).all() and torch.isfinite(dbeta).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_one_segment_does_not_reach_another(m, bad):
    import torch
    rng = np.random.default_rng(6)
    x, _ = tensors(rng, 3000, 32, "float32")
    dy = torch.randn(3000, 32, device="cuda")
    p = torch.tensor([0, 1000, 2001, 3000], dtype=torch.int32, device="cuda")
    one, zero = torch.ones(32, device="cuda"), torch.zeros(32, device="cuda")
    y, mean, rstd = m.egnn_group_norm(x, 4, one, zero, ptr=p)
    dx, _, _ = m.egnn_group_norm_backward(x, dy, mean, rstd, 4, one, zero, ptr=p)
    x2 = x.clone()
    x2[1500, 3] = bad
    y2, mean2, rstd2 = m.egnn_group_norm(x2, 4, one, zero, ptr=p)
    dx2, _, _ = m.egnn_group_norm_backward(x2, dy, mean2, rstd2, 4, one, zero, ptr=p)
    rows = torch.cat([torch.arange(1000), torch.arange(2001, 3000)]).cuda()
    assert torch.equal(y2[rows], y[rows]) and torch.equal(dx2[rows], dx[rows])
    assert torch.isnan(y2[1000:2001, :8]).any() and torch.isfinite(y2[1000:2001, 8:]).all()


def test_pointers_out_of_range_are_clamped(m):
    import torch
    rng = np.random.default_rng(7)
    x, _ = tensors(rng, 100, 16, "float32")
    one, zero = torch.ones(16, device="cuda"), torch.zeros(16, device="cuda")
    good = m.egnn_group_norm(x, 4, one, zero, ptr=torch.tensor([0, 40, 100], dtype=torch.int32, device="cuda"))
    far = m.egnn_group_norm(x, 4, one, zero, ptr=torch.tensor([-7, 40, 10 ** 9], dtype=torch.int32, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(good, far))


def test_no_rows(m):
    import torch
    x = torch.empty((0, 16), device="cuda")
    one, zero = torch.ones(16, device="cuda"), torch.zeros(16, device="cuda")
    p = torch.zeros(4, dtype=torch.int32, device="cuda")
    y, mean, rstd = m.egnn_group_norm(x, 4, one, zero, ptr=p)
    assert y.shape == (0, 16) and not mean.any() and not rstd.any() and mean.shape == (3, 4)
    dx, dgamma, dbeta = m.egnn_group_norm_backward(x, x, mean, rstd, 4, one, zero, ptr=p)
    assert not dgamma.any() and not dbeta.any()


def test_same_bits_again_on_another_stream_and_in_a_graph(m):
    import torch
    rng = np.random.default_rng(8)
    x, _ = tensors(rng, 30000, 64, "float32")
    x = x.contiguous()
    dy = torch.randn_like(x)
    p = torch.tensor([0, 10, 20000, 30000], dtype=torch.int32, device="cuda")
    ga, be = torch.randn(64, device="cuda"), torch.randn(64, device="cuda")
    y, mean, rstd = m.egnn_group_norm(x, 8, ga, be, ptr=p)
    want = (y, mean, rstd, *m.egnn_group_norm_backward(x, dy, mean, rstd, 8, ga, be, ptr=p))
    ws = torch.empty(m.egnn_group_norm_workspace_bytes(30000, 3, 64, 8), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(t) for t in want]

    def both():
        m.egnn_group_norm(x, 8, ga, be, ptr=p, y=outs[0], mean=outs[1], rstd=outs[2], ws=ws)
        m.egnn_group_norm_backward(x, dy, outs[1], outs[2], 8, ga, be, ptr=p, dx=outs[3], dgamma=outs[4], dbeta=outs[5], ws=ws)

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in outs:
            t.fill_(7.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
