"""Orthogonalised updates and the optimiser's step against oracle/block_oracle.py (fp64).

Tolerances, relative in the 2-norm.  A step x -> a x + b g x + c g^2 x rounds each of its three terms a few times: 8 roundings of
(a + |b| + |c|) = 10.25 parts of x, five steps: 5 * 8 * 10.25 * 2^-24 = 2.4e-5 where the steps do not amplify (a matrix of full rank grows with
its errors).  Of a matrix of low rank the errors in the empty directions grow by a = 3.4445 a step while the matrix does not: times 3.4445^4.
Outputs in fewer bits add half a step of their type; wide bfloat16 updates are made from operands of 11 bits (four half steps of 2^-12 = 2^-10)."""
import numpy as np
import pytest

from oracle import block_oracle as K

pytestmark = pytest.mark.gpu
FULL = 5 * 8 * 10.25 * 2.0 ** -24
TOL = {"float32": FULL, "float16": FULL + 2.0 ** -11, "bfloat16": FULL + 2.0 ** -8 + 2.0 ** -10}


@pytest.fixture(scope="module")
def m():
    from paper_2507_03840_amd import binding as B
    return B.Egnn(2, 32, 16, 10.0, 200.0)


def off(got, want):
    d = got.double().cpu().numpy() - want
    return max(np.linalg.norm(d[i]) / max(np.linalg.norm(want[i]), 1e-300) for i in range(d.shape[0]))


def random(rng, *shape):
    """A few strong directions over many weak ones, as gradients have."""
    b, n, m = shape
    r = max(1, min(n, m) // 8)
    return 1e-3 * (rng.standard_normal(shape) + 2.0 * rng.standard_normal((b, n, r)) @ rng.standard_normal((b, r, m)))


SHAPES = [(1, 1, 1), (3, 1, 7), (2, 7, 1), (2, 5, 5), (15, 32, 32), (2, 31, 33), (3, 64, 64), (2, 65, 64), (1, 64, 65), (2, 8, 300), (2, 700, 64),
          (1, 130, 1001), (2, 100, 90), (1, 96, 128), (3, 129, 127), (1, 320, 480), (1, 300, 301), (1, 640, 257), (1, 2048, 20)]


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalise(m, shape, dtype):
    import torch
    g = torch.from_numpy(random(np.random.default_rng([1, *shape]), *shape)).to(getattr(torch, dtype)).cuda()
    y = m.egnn_orthogonalise(g)
    e = off(y, K.orthogonalise(g.double().cpu().numpy()))
    print(shape, dtype, "off by %.2e" % e)
    assert y.dtype == g.dtype and e <= TOL[dtype]


@pytest.mark.parametrize("steps", [1, 2, 3, 7])
@pytest.mark.parametrize("shape", [(2, 20, 20), (1, 64, 500), (1, 200, 150)])
def test_number_of_steps(m, shape, steps):
    import torch
    g = torch.from_numpy(random(np.random.default_rng([2, *shape]), *shape)).float().cuda()
    assert off(m.egnn_orthogonalise(g, steps=steps), K.orthogonalise(g.double().cpu().numpy(), steps)) <= FULL * max(1.0, steps / 5)


@pytest.mark.parametrize("shape", [(1, 24, 24), (1, 40, 400), (1, 200, 300)])
def test_low_rank(m, shape):
    import torch
    rng = np.random.default_rng([3, *shape])
    g = torch.from_numpy(rng.standard_normal((1, shape[1], 2)) @ rng.standard_normal((1, 2, shape[2]))).float().cuda()
    assert off(m.egnn_orthogonalise(g), K.orthogonalise(g.double().cpu().numpy())) <= FULL * 3.4445 ** 4


@pytest.mark.parametrize("shape", [(2, 16, 16), (2, 64, 200), (2, 150, 100)])
@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e18])
def test_scales(m, shape, scale):
    """The norm neither overflows nor underflows; a norm near 1e-7 and below shrinks the result as the formula says."""
    import torch
    rng = np.random.default_rng([4, *shape])
    g = torch.from_numpy(rng.standard_normal(shape) * scale).float().cuda()
    want = K.orthogonalise(g.double().cpu().numpy())
    got = m.egnn_orthogonalise(g)
    assert torch.isfinite(got).all()
    if scale > 1e-20:
        assert off(got, want) <= 2 * FULL
    else:      # x is about 1e-21 everywhere: below what half-precision pieces of a matrix of norm 1 hold
        assert np.abs(got.double().cpu().numpy()).max() <= 1e-6


def test_zero_and_batch_apart(m):
    """A matrix of zeros gives zeros; one with a NaN does not reach its neighbours."""
    import torch
    for shape in ((3, 20, 20), (3, 64, 300), (3, 150, 200)):
        g = torch.from_numpy(random(np.random.default_rng([5, *shape]), *shape)).float().cuda()
        want = m.egnn_orthogonalise(g)
        g[1] = 0.0
        y = m.egnn_orthogonalise(g)
        assert not y[1].any() and torch.equal(y[0], want[0]) and torch.equal(y[2], want[2])
        g[1, 2, 3] = float("nan")
        y = m.egnn_orthogonalise(g)
        assert torch.isnan(y[1]).all() and torch.equal(y[0], want[0]) and torch.equal(y[2], want[2])


@pytest.mark.parametrize("shape", [(15, 32, 32), (3, 700, 64), (1, 64, 64), (2, 200, 300), (1, 300, 120), (4, 10, 1)])
def test_muon_step(m, shape):
    import torch
    rng = np.random.default_rng([6, *shape])
    dev = lambda a: torch.from_numpy(a).float().cuda()
    W, g, mom = dev(rng.standard_normal(shape) * shape[2] ** -0.5), dev(random(rng, *shape)), dev(random(rng, *shape))
    f = lambda t: t.double().cpu().numpy()
    rW, rm = K.muon_step(f(W), f(g), f(mom), 0.02, 0.95, 0.01)
    W2, m2 = m.egnn_muon_step(W, g, mom, 0.02, beta=0.95, weight_decay=0.01, W_out=torch.empty_like(W), momentum_out=torch.empty_like(W))
    assert np.abs(f(m2) - rm).max() <= 4 * 2.0 ** -24 * np.abs(rm).max()
    o = np.linalg.norm(K.orthogonalise(f(g) + 0.95 * rm)) * 0.02 * max(1.0, shape[1] / shape[2]) ** 0.5
    assert np.linalg.norm(f(W2) - rW) <= 2 * FULL * o + 3 * 2.0 ** -24 * np.linalg.norm(rW)
    W3, m3 = m.egnn_muon_step(W, g, mom, 0.02, beta=0.95, weight_decay=0.01)     # in place
    assert W3 is W and m3 is mom and torch.equal(W, W2) and torch.equal(mom, m2)


def test_no_matrices_and_in_place(m):
    import torch
    assert m.egnn_orthogonalise(torch.empty((0, 4, 5), device="cuda")).shape == (0, 4, 5)
    for shape in ((2, 30, 20), (1, 100, 200)):
        g = torch.from_numpy(random(np.random.default_rng([7, *shape]), *shape)).float().cuda()
        y = m.egnn_orthogonalise(g)
        assert m.egnn_orthogonalise(g, y=g) is g and torch.equal(g, y)


@pytest.mark.parametrize("shape", [(15, 32, 32), (3, 400, 64), (1, 200, 300)])
def test_same_bits_again_on_another_stream_and_in_a_graph(m, shape):
    import torch
    rng = np.random.default_rng([8, *shape])
    dev = lambda a: torch.from_numpy(a).float().cuda()
    W, g, mom = dev(rng.standard_normal(shape)), dev(random(rng, *shape)), dev(random(rng, *shape))
    new = lambda: (torch.empty_like(W), torch.empty_like(W))
    w, n = new()
    want = m.egnn_muon_step(W, g, mom, 0.02, W_out=w, momentum_out=n)
    ws = torch.empty(m.egnn_orthogonalise_workspace_bytes(*shape), dtype=torch.uint8, device="cuda")
    outs = new()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        m.egnn_muon_step(W, g, mom, 0.02, W_out=outs[0], momentum_out=outs[1], ws=ws)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.egnn_muon_step(W, g, mom, 0.02, W_out=outs[0], momentum_out=outs[1], ws=ws)
    for _ in range(3):
        for t in outs:
            t.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("shape", [(5, 300, 700), (3, 1000, 650), (2, 1290, 1100)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_wide_tiles(m, shape, dtype):
    """Enough tiles of 128 for half the compute units; sides that are no multiples of them."""
    import torch
    g = torch.from_numpy(random(np.random.default_rng([9, *shape]), *shape)).to(getattr(torch, dtype)).cuda()
    e = off(m.egnn_orthogonalise(g), K.orthogonalise(g.double().cpu().numpy()))
    print(shape, dtype, "off by %.2e" % e)
    assert e <= TOL[dtype]


@pytest.mark.parametrize("shape", [(1, 20, 17000), (1, 17000, 50)])
def test_more_columns_than_slabs(m, shape):
    """A workgroup takes several slabs in turn."""
    import torch
    g = torch.from_numpy(random(np.random.default_rng([10, *shape]), *shape)).float().cuda()
    assert off(m.egnn_orthogonalise(g), K.orthogonalise(g.double().cpu().numpy())) <= FULL
    W, mom = torch.randn(shape, device="cuda"), torch.zeros(shape, device="cuda")
    f = lambda t: t.double().cpu().numpy()
    rW, rm = K.muon_step(f(W), f(g), f(mom), 0.02, 0.95, 0.01)
    W2, m2 = m.egnn_muon_step(W, g, mom, 0.02, beta=0.95, weight_decay=0.01)
    assert np.abs(f(m2) - rm).max() <= 4 * 2.0 ** -24 * np.abs(rm).max()
    o = np.linalg.norm(K.orthogonalise(f(g) + 0.95 * rm)) * 0.02 * max(1.0, shape[1] / shape[2]) ** 0.5
    assert np.linalg.norm(f(W2) - rW) <= 2 * FULL * o + 3 * 2.0 ** -24 * np.linalg.norm(rW)


@pytest.mark.parametrize("shape", [(2, 21, 30), (2, 500, 44), (1, 130, 90)])
def test_alignment(m, shape):
    """Matrices that begin at any element of a larger buffer give the same numbers (to rounding) as aligned ones."""
    import torch
    n = int(np.prod(shape))
    for dtype in (torch.float32, torch.bfloat16):
        g = torch.from_numpy(random(np.random.default_rng([11, *shape]), *shape)).to(dtype).cuda()
        want = m.egnn_orthogonalise(g)
        room, out = torch.zeros(n + 8, dtype=dtype, device="cuda"), torch.full((n + 8,), 7.0, dtype=dtype, device="cuda")
        for at in (1, 2, 3):
            room[at:at + n] = g.reshape(-1)
            y = m.egnn_orthogonalise(room[at:at + n].view(shape), y=out[at:at + n].view(shape))
            assert off(y, want.double().cpu().numpy()) <= TOL["float32" if dtype == torch.float32 else "bfloat16"]
            assert (out[:at] == 7.0).all() and (out[at + n:] == 7.0).all()
            out.fill_(7.0)
