"""Rows in groups, grouped linear maps and their adjoint against oracle/block_oracle.py (fp64).

Tolerances.  A sum of k products in fp32, in any order, is off by at most (k + 8) roundings of the sum of its absolute terms (the 8 cover
products of fp32 operands from pieces, their dropped parts and the bias); the output's own rounding is half a step of its type."""
import numpy as np
import pytest

from oracle import block_oracle as K

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
FLOOR = {"float32": 1e-37, "float16": 2.0 ** -25, "bfloat16": 1e-37}


@pytest.fixture(scope="module")
def m():
    from paper_2507_03840_amd import binding as B
    return B.Egnn(2, 32, 16, 10.0, 200.0)


@pytest.mark.parametrize("n,groups,lmax", [(0, 3, -1), (0, 2, 2), (1, 1, -1), (1, 4, 3), (63, 2, -1), (64, 64, -1), (1000, 3, 4), (1025, 7, -1),
                                           (5001, 1, -1), (5001, 1024, -1), (3000, 1000, 1), (70000, 5, 1), (600000, 33, -1), (40000, 64, 0)])
def test_group_rows(m, n, groups, lmax):
    import torch
    key = np.random.default_rng([1, n, groups]).integers(-2, groups + 2, n).astype(np.int32)
    ptr, perm = m.egnn_group_rows(torch.from_numpy(key).cuda(), groups, lmax=lmax)
    rptr, rperm = K.group_rows(key, groups, lmax)
    assert np.array_equal(ptr.cpu().numpy(), rptr) and np.array_equal(perm.cpu().numpy(), rperm)


def test_group_rows_sorted_and_single_keys(m):
    import torch
    for key in (np.sort(np.random.default_rng(2).integers(0, 9, 4000)), np.full(3000, 4), np.arange(3000)[::-1] % 9):
        key = key.astype(np.int32)
        ptr, perm = m.egnn_group_rows(torch.from_numpy(key).cuda(), 9)
        rptr, rperm = K.group_rows(key, 9)
        assert np.array_equal(ptr.cpu().numpy(), rptr) and np.array_equal(perm.cpu().numpy(), rperm)


def data(rng, n, k, out, groups, dtype, empty=()):
    import torch
    t = getattr(torch, dtype)
    there = [g for g in range(groups) if g not in empty]
    key = rng.choice(there, n)
    ptr, perm = K.group_rows(key, groups)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()
    x, W, dy = dev(rng.standard_normal((n, k)), t), dev(rng.standard_normal((groups, out, k)) * k ** -0.5, t), dev(rng.standard_normal((n, out)), t)
    return x, W, dy, dev(rng.standard_normal((groups, out)), torch.float32), dev(ptr, torch.int32), dev(perm, torch.int32), ptr, perm


def close(got, want, size, terms, u, floor):
    got = got.double().cpu().numpy()
    rows = ~np.isnan(want)
    off = np.abs(got - want)[rows] - (u * np.abs(want) + floor + (terms + 8) * U32 * size)[rows]
    assert np.isfinite(got[rows]).all() and off.max(initial=-1) <= 0, off.max()


def check(m, n, k, out, groups, dtype, empty=(), with_perm=True, seed=0):
    rng = np.random.default_rng([seed, n, k, out, groups])
    x, W, dy, bias, ptr, perm, hptr, hperm = data(rng, n, k, out, groups, dtype, empty)
    if not with_perm:
        perm = hperm = None
    f = lambda t: t.double().cpu().numpy()
    u, fl = HALF_STEP[dtype], FLOOR[dtype]
    y = m.egnn_grouped_linear(x, W, ptr, perm=perm, bias=bias)
    ry, sy = K.grouped_linear(f(x), f(W), hptr, hperm, f(bias))
    close(y, ry, sy, k, u, fl)
    y = m.egnn_grouped_linear(x, W, ptr, perm=perm)
    ry, sy = K.grouped_linear(f(x), f(W), hptr, hperm)
    close(y, ry, sy, k, u, fl)
    dx, dW, db = m.egnn_grouped_linear_backward(x, W, dy, ptr, perm=perm)
    rdx, rdW, rdb, sx, sW, sb = K.grouped_linear_backward(f(x), f(W), f(dy), hptr, hperm)
    close(dx, rdx, sx, out, u, fl)
    most = int(np.diff(hptr).max(initial=0))
    close(dW, rdW, sW, most, U32, 1e-37)
    close(db, rdb, sb, most, U32, 1e-37)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("k,out", [(1, 1), (3, 5), (8, 8), (16, 16), (17, 64), (64, 17), (64, 64), (32, 128), (77, 100), (100, 77), (129, 65), (256, 31),
                                   (96, 320), (514, 130)])
def test_shapes(m, k, out, dtype):
    for n, groups in ((1, 1), (7, 3), (200, 2), (513, 5)):
        check(m, n, k, out, groups, dtype)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("n,groups,empty", [(1, 9, range(8)), (64, 3, [1]), (65, 64, []), (129, 200, range(0, 200, 3)), (1000, 4, [0, 3]),
                                            (2000, 700, []), (20000, 3, [2])])
def test_groups(m, n, groups, empty, dtype):
    check(m, n, 24, 40, groups, dtype, empty=list(empty))
    check(m, n, 64, 64, groups, dtype, empty=list(empty), with_perm=False)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_larger(m, dtype):
    check(m, 5000, 512, 384, 3, dtype)
    check(m, 30000, 64, 64, 15, dtype, seed=1)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("planes", [2, 3])
def test_rows_inside_larger_tensors(m, dtype, planes):
    """x, dy and the outputs are planes of larger tensors, of odd lengths too; the other planes are left alone."""
    import torch
    for n, k, out in ((300, 32, 48), (111, 33, 7)):
        rng = np.random.default_rng([5, k])
        x, W, dy, bias, ptr, perm, hptr, hperm = data(rng, n, k, out, 4, dtype)
        y = m.egnn_grouped_linear(x, W, ptr, perm=perm, bias=bias)
        dx, dW, db = m.egnn_grouped_linear_backward(x, W, dy, ptr, perm=perm)
        wide = lambda t: torch.full((n, planes, t.shape[1]), 3.0, dtype=t.dtype, device="cuda")
        X, D, Y, G = wide(x), wide(dy), wide(y), wide(dx)
        X[:, 1], D[:, 1] = x, dy
        m.egnn_grouped_linear(X[:, 1], W, ptr, perm=perm, bias=bias, y=Y[:, 1])
        _, dW2, db2 = m.egnn_grouped_linear_backward(X[:, 1], W, D[:, 1], ptr, perm=perm, dx=G[:, 1])
        assert torch.equal(Y[:, 1], y) and torch.equal(G[:, 1], dx) and torch.equal(dW2, dW) and torch.equal(db2, db)
        assert (Y[:, 0] == 3.0).all() and (G[:, 0] == 3.0).all() and (Y[:, 2:] == 3.0).all() and (G[:, 2:] == 3.0).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_far_magnitudes(m, dtype):
    """Rows and matrices of very small and very large numbers keep their relative accuracy (no common scale)."""
    import torch
    rng = np.random.default_rng(6)
    x, W, dy, bias, ptr, perm, hptr, hperm = data(rng, 400, 64, 64, 2, dtype)
    scale = torch.exp2(torch.randint(-40, 40, (400, 1), device="cuda").float()).to(x.dtype)
    x, dy = x * scale, dy / scale
    f = lambda t: t.double().cpu().numpy()
    ry, sy = K.grouped_linear(f(x), f(W), hptr, hperm)
    close(m.egnn_grouped_linear(x, W, ptr, perm=perm), ry, sy, 64, HALF_STEP[dtype], 1e-30)
    dx, dW, db = m.egnn_grouped_linear_backward(x, W, dy, ptr, perm=perm)
    rdx, rdW, rdb, sx, sW, sb = K.grouped_linear_backward(f(x), f(W), f(dy), hptr, hperm)
    close(dx, rdx, sx, 64, HALF_STEP[dtype], 1e-30)
    close(dW, rdW, sW, 400, U32, 1e-30)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_one_row_does_not_reach_another(m, dtype, bad):
    import torch
    rng = np.random.default_rng(7)
    x, W, dy, bias, ptr, perm, hptr, hperm = data(rng, 300, 40, 24, 3, dtype)
    y = m.egnn_grouped_linear(x, W, ptr, perm=perm)
    dx, dW, db = m.egnn_grouped_linear_backward(x, W, dy, ptr, perm=perm)
    row = int(hperm[hptr[1]])     # the first row of group 1: it shares tiles with the end of group 0
    x2, dy2 = x.clone(), dy.clone()
    x2[row, 3], dy2[row, 2] = bad, bad
    y2 = m.egnn_grouped_linear(x2, W, ptr, perm=perm)
    dx2, dW2, db2 = m.egnn_grouped_linear_backward(x2, W, dy2, ptr, perm=perm)
    others = torch.arange(300, device="cuda") != row
    assert torch.equal(y2[others], y[others]) and torch.equal(dx2[others], dx[others])
    assert not torch.isfinite(y2[row]).any() and not torch.isfinite(dx2[row]).any()
    for g in (0, 2):
        assert torch.equal(dW2[g], dW[g]) and torch.equal(db2[g], db[g])
    assert not torch.isfinite(dW2[1][2]).any() and not torch.isfinite(dW2[1][:, 3]).any() and not torch.isfinite(db2[1][2])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_infinite_weights_stay_in_their_column(m, dtype):
    import torch
    rng = np.random.default_rng(8)
    x, W, dy, bias, ptr, perm, _, _ = data(rng, 200, 32, 48, 2, dtype)
    y = m.egnn_grouped_linear(x, W, ptr, perm=perm)
    W2 = W.clone()
    W2[1, 5, 7] = float("inf")
    y2 = m.egnn_grouped_linear(x, W2, ptr, perm=perm)
    keep = torch.ones(48, dtype=torch.bool, device="cuda")
    keep[5] = False
    assert torch.equal(y2[:, keep], y[:, keep])


def test_rows_of_no_group_and_pointers_out_of_range(m):
    import torch
    rng = np.random.default_rng(9)
    x, W, dy, bias, ptr, perm, hptr, hperm = data(rng, 100, 16, 16, 3, "float32")
    y = torch.full((100, 16), 9.0, device="cuda")
    short = ptr.clone()
    short[-1] = short[-2]
    m.egnn_grouped_linear(x, W, short, perm=perm, y=y)
    left = torch.from_numpy(hperm[hptr[2]:].astype(np.int64)).cuda()
    assert (y[left] == 9.0).all()
    far = ptr.clone()
    far[0], far[-1] = -5, 10 ** 9
    assert torch.equal(m.egnn_grouped_linear(x, W, far, perm=perm), m.egnn_grouped_linear(x, W, ptr, perm=perm))
    lost = perm.clone()
    lost[hptr[1]] = 10 ** 6       # clamped to the last row
    assert torch.isfinite(m.egnn_grouped_linear(x, W, ptr, perm=lost, y=torch.zeros_like(y))).all()


def test_no_rows(m):
    import torch
    W = torch.randn(3, 5, 4, device="cuda")
    x, dy = torch.empty((0, 4), device="cuda"), torch.empty((0, 5), device="cuda")
    ptr, perm = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    assert m.egnn_grouped_linear(x, W, ptr, perm=perm).shape == (0, 5)
    dx, dW, db = m.egnn_grouped_linear_backward(x, W, dy, ptr, perm=perm)
    assert dx.shape == (0, 4) and not dW.any() and not db.any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_same_bits_again_on_another_stream_and_in_a_graph(m, dtype):
    import torch
    rng = np.random.default_rng(10)
    n, k, out, groups = 5000, 64, 96, 6
    x, W, dy, bias, _, _, _, _ = data(rng, n, k, out, groups, dtype)
    key = torch.from_numpy(rng.integers(0, groups, n).astype(np.int32)).cuda()
    ptr, perm = m.egnn_group_rows(key, groups)
    want = (ptr, perm, m.egnn_grouped_linear(x, W, ptr, perm=perm, bias=bias), *m.egnn_grouped_linear_backward(x, W, dy, ptr, perm=perm))
    ws = torch.empty(max(m.egnn_grouped_linear_workspace_bytes(n, groups, k, out), m.egnn_group_rows_workspace_bytes(n, groups)),
                     dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(t) for t in want]

    def both():
        m.egnn_group_rows(key, groups, ptr=outs[0], perm=outs[1], ws=ws)
        m.egnn_grouped_linear(x, W, outs[0], perm=outs[1], bias=bias, y=outs[2])
        m.egnn_grouped_linear_backward(x, W, dy, outs[0], perm=outs[1], dx=outs[3], dW=outs[4], db=outs[5], ws=ws)

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
            t.fill_(0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("n,k,out,groups,empty", [(90001, 61, 37, 3, []), (80000, 64, 64, 200, range(0, 200, 7)), (100003, 9, 50, 2, [0])])
def test_many_rows_of_small_matrices(m, n, k, out, groups, empty, dtype):
    """The way of many rows: matrices in registers."""
    check(m, n, k, out, groups, dtype, empty=list(empty))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_wide_tiles_of_ragged_groups(m, dtype):
    """Enough tiles for the wide kernels: groups of a few rows, of none, odd rows and columns; then one group of nearly all rows."""
    check(m, 900, 203, 259, 90, dtype, empty=[0, 7, 89])
    check(m, 905, 264, 200, 90, dtype, with_perm=False)
    check(m, 4000, 136, 1000, 40, dtype, empty=list(range(1, 38)))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_groups_longer_than_the_row_numbers_kept(m, dtype):
    """More than 2,048 rows of one group in one workgroup of the weight gradient."""
    check(m, 6001, 1024, 1000, 2, dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("k,out", [(40, 24), (64, 64), (200, 140)])
def test_gradients_one_at_a_time(m, k, out, dtype):
    """Any of dx, dW, db may be left out of the C call; the others keep their values."""
    import torch
    rng = np.random.default_rng([12, k])
    for n in (300, 90000):
        x, W, dy, bias, ptr, perm, hptr, hperm = data(rng, n, k, out, 3, dtype)
        want = m.egnn_grouped_linear_backward(x, W, dy, ptr, perm=perm)
        ws = torch.empty(max(256, m.egnn_grouped_linear_workspace_bytes(n, 3, k, out)), dtype=torch.uint8, device="cuda")
        for keep in range(1, 7):
            outs = [torch.full_like(t, 3.0) if keep >> i & 1 else None for i, t in enumerate(want)]
            at = [None if t is None else t.data_ptr() for t in outs]
            rc = m.lib.egnn_grouped_linear_backward(
                m.ctx, {"float32": 0, "bfloat16": 2}[dtype], x.data_ptr() if keep & 2 else None, k, W.data_ptr() if keep & 1 else None, dy.data_ptr(), out, n, k, out,
                ptr.data_ptr(), perm.data_ptr(), 3, at[0], k, at[1], at[2], ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
            assert rc == 0
            assert all(t is None or torch.equal(t, w) for t, w in zip(outs, want)), keep


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("k,out", [(24, 40), (128, 136)])
def test_offsets_past_32_bits(m, k, out, dtype):
    """Rows 100,000 values apart: the last lie behind 2^32 values."""
    import torch
    n = 50000
    x, W, dy, bias, ptr, perm, _, _ = data(np.random.default_rng([6, k]), n, k, out, 3, dtype)
    whole = torch.empty((n, 100000), dtype=x.dtype, device="cuda")
    X, G, D, Y = (whole[:, 1000 * i:1000 * i + c] for i, c in enumerate((k, k, out, out)))
    X.copy_(x), D.copy_(dy)
    y = m.egnn_grouped_linear(x, W, ptr, perm=perm, bias=bias)
    dx, dW, db = m.egnn_grouped_linear_backward(x, W, dy, ptr, perm=perm)
    m.egnn_grouped_linear(X, W, ptr, perm=perm, bias=bias, y=Y)
    _, dW2, db2 = m.egnn_grouped_linear_backward(X, W, D, ptr, perm=perm, dx=G)
    assert torch.equal(X, x) and torch.equal(D, dy)
    assert torch.equal(Y, y) and torch.equal(G, dx) and torch.equal(dW2, dW) and torch.equal(db2, db)
