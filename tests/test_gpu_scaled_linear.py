"""Products of rows and matrices in 8-bit codes with scales against oracle/residual_oracle.py and oracle/block_oracle.py (fp64).

Tolerances.  fp32 and fp16 results: products of codes are exact; a term passes at most 16 sums of eight inside its block of 128, one per block and two
more (scale's sum, bias), each off by a rounding, or two if cut off, of the sum of magnitudes S: 2 (18 + K / 128) U32 S, and u of the result.
bf16 results: the 8-bit instruction cuts seven of eight products off at 2^-13 of the largest, and its sums of eight are added one after the
other: 7 * 2^-13 S + 2 (2 + K / 8) U32 S, and u of the result.  Where that hides a missing term, values are chosen that every step holds
exactly: then results are equal."""
import numpy as np
import pytest

from oracle import block_oracle as K, residual_oracle as R
from tests.residual_util import FLOOR, HALF_STEP, U32, values

pytestmark = pytest.mark.gpu
TYPES = ["float32", "float16", "bfloat16"]


@pytest.fixture(scope="module")
def m():
    from paper_2507_03840_amd import binding as B
    return B.Egnn(2, 32, 16, 10.0, 200.0)


def rows_on_device(code, e):
    import torch
    from paper_2507_03840_amd import binding as B
    q, s = B.empty_codes(code.shape)
    q.as_strided((*code.shape[:-1], q.stride(-2)), q.stride()).view(torch.uint8).zero_()
    q.view(torch.uint8).copy_(torch.from_numpy(code))
    s.view(torch.uint8).copy_(torch.from_numpy((e + 127).astype(np.uint8)))
    return q, s


def matrices_on_device(code, e):
    import torch
    from paper_2507_03840_amd import binding as B
    q, s = B.empty_matrix_codes(code.shape)
    q.as_strided((*code.shape[:-1], q.stride(-2)), q.stride()).view(torch.uint8).zero_()
    q.view(torch.uint8).copy_(torch.from_numpy(code))
    s.view(torch.uint8).copy_(torch.from_numpy((e + 127).astype(np.uint8)))
    return q, s


def random_operands(rng, n, k, groups, out, spread=0):
    """Codes of normal values, exponents of any size up to `spread` in either direction."""
    x, W = rng.standard_normal((n, k)), rng.standard_normal((groups, out, k))
    q, e, _ = R.quantise_rows(x)
    w, we = R.quantise_matrices(W)
    return q, e + rng.integers(-spread, spread + 1, e.shape), w, we + rng.integers(-spread, spread + 1, we.shape)


def bound(y, size, k, dtype):
    off = 2 * (18 + k / 128) * U32 if dtype != "bfloat16" else 7 * 2.0 ** -13 + 2 * (2 + k / 8) * U32
    return off * size + HALF_STEP[dtype] * np.abs(y) + FLOOR[dtype]


def check(m, n, k, out, dtype, groups=1, ptr=None, perm=None, bias=True, spread=0, seed=0):
    import torch
    rng = np.random.default_rng([seed, n, k, out])
    q, e, w, we = random_operands(rng, n, k, groups, out, spread)
    b = rng.standard_normal((groups, out)).astype(np.float32) if bias else None
    t = lambda a: None if a is None else torch.from_numpy(np.asarray(a, np.int32)).cuda()
    y = torch.full((n, out), 77.0, dtype=getattr(torch, dtype), device="cuda")
    m.egnn_scaled_linear(*rows_on_device(q, e), *matrices_on_device(w, we), ptr=t(ptr), perm=t(perm), bias=None if b is None else torch.from_numpy(b).cuda(), y=y)
    ry, size = K.grouped_linear(R.values_of_rows(q, e), R.values_of_matrices(w, we), [0, n] if ptr is None else ptr, perm, b)
    got, there = values(y), ~np.isnan(ry).all(1)
    assert (np.abs(got - ry) <= bound(ry, size, k, dtype))[there].all()
    assert (got[~there] == 77.0).all()
    if n * out >= 2000 and not spread and k >= 64 and there.all():           # as a whole: the rounding of the result, and 1.5e-5 beside it
        assert np.linalg.norm(got - ry) <= (2 * HALF_STEP[dtype] / 3 ** 0.5 + 3e-5) * np.linalg.norm(ry)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [1, 15, 16, 17, 32, 33, 64, 100, 127, 128, 129, 144, 256, 300, 1000])
def test_contractions(m, k, dtype):
    for n, out in ((1, 40), (70, 33), (200, 64)):
        check(m, n, k, out, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,out", [(1, 1), (2, 7), (15, 16), (16, 17), (17, 130), (33, 300), (63, 8), (64, 64), (65, 128), (127, 129), (128, 256), (129, 257), (300, 31),
                                   (1000, 200), (2500, 136)])
def test_sides(m, n, out, dtype):
    check(m, n, 64, out, dtype)
    check(m, n, 272, out, dtype, bias=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 3, 16, 20, 64])
@pytest.mark.parametrize("k,out", [(2048, 48), (4096, 256), (8200, 20), (20000, 5)])
def test_few_rows_and_long_contractions(m, k, out, n, dtype):
    check(m, n, k, out, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_larger_products(m, dtype):
    check(m, 1300, 640, 520, dtype)
    check(m, 700, 1104, 900, dtype)


GROUPS = [([0, 10, 10, 40, 90], 90), ([0, 0, 0, 90], 90), ([5, 20, 60, 60], 90), ([0, 64, 128, 192, 200], 200), ([0, 1, 2, 3, 4, 300], 300), (list(range(0, 301, 3)), 300)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ptr,n", GROUPS)
def test_groups(m, ptr, n, dtype):
    """Empty groups, rows before the first and behind the last left as they are, rows in any order."""
    rng = np.random.default_rng(n)
    check(m, n, 64, 64, dtype, len(ptr) - 1, ptr)
    check(m, n, 70, 33, dtype, len(ptr) - 1, ptr, rng.permutation(n))
    check(m, n, 200, 130, dtype, len(ptr) - 1, ptr, rng.permutation(n), bias=False)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_more_groups_than_a_wave(m, dtype):
    rng = np.random.default_rng(8)
    ptr = np.concatenate([[0], np.cumsum(rng.integers(0, 7, 333))])
    check(m, int(ptr[-1]), 48, 20, dtype, 333, ptr, rng.permutation(int(ptr[-1])))
    ptr = np.concatenate([np.zeros(400, int), np.full(300, 500)])
    check(m, 500, 32, 16, dtype, 699, ptr)


def check_large(m, n, k, out, dtype, groups=1, ptr=None, perm=None, seed=0):
    """check() with values and an oracle (fp64 products of the values of the codes) made on the device."""
    import torch
    torch.manual_seed(seed)
    a = m.egnn_quantise_rows(torch.randn(n, k, device="cuda") * torch.rand(n, 1, device="cuda"))
    b = m.egnn_quantise_matrices(torch.randn(groups, out, k, device="cuda"))[:2]
    bias = torch.randn(groups, out, device="cuda")
    x = a[0].double() * a[1].double().repeat_interleave(128, 1)[:, :k]
    W = b[0].double() * b[1].double().repeat_interleave(128, 2)[:, :, :k].repeat_interleave(128, 1)[:, :out]
    t = lambda v: None if v is None else torch.as_tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    y = torch.full((n, out), 77.0, dtype=getattr(torch, dtype), device="cuda")
    m.egnn_scaled_linear(*a, *b, ptr=t(ptr), perm=t(perm), bias=bias, y=y)
    order, at = torch.arange(n, device="cuda") if perm is None else t(perm).long(), [0, n] if ptr is None else [int(v) for v in ptr]
    seen = torch.zeros(n, dtype=torch.bool, device="cuda")
    off = 2 * (18 + k / 128) * U32 if dtype != "bfloat16" else 7 * 2.0 ** -13 + 2 * (2 + k / 8) * U32
    for g in range(groups):
        rows = order[at[g]:at[g + 1]]
        seen[rows] = True
        ry = x[rows] @ W[g].t() + bias[g]
        size = x[rows].abs() @ W[g].abs().t() + bias[g].abs()
        far = (y[rows].double() - ry).abs()
        assert (far <= off * size + HALF_STEP[dtype] * ry.abs() + FLOOR[dtype]).all()
        if len(rows) > 100:
            assert far.norm() <= (2 * HALF_STEP[dtype] / 3 ** 0.5 + 3e-5) * ry.norm()
    assert (y[~seen] == 77.0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k,out", [(20001, 300, 520), (3600, 2100, 3400), (4097, 2048, 4090), (2050, 700, 2000), (5120, 136, 5000)])
def test_many_tiles(m, n, k, out, dtype):
    check_large(m, n, k, out, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k,out,ptr", [(3000, 200, 300, [0, 0, 1, 700, 700, 2999]), (30001, 200, 260, [7, 7, 5000, 5001, 12345, 29000, 29000, 30001]),
                                         (4500, 2100, 3300, [0, 2001, 4500]), (70000, 64, 64, [0, 10, 30000, 30000, 69999]), (5000, 130, 40, [0, 2500, 5000])])
def test_many_tiles_in_groups(m, n, k, out, ptr, dtype):
    """The last rows of a group and the first of the next in one tile's reach; rows in any order and in their own."""
    check_large(m, n, k, out, dtype, len(ptr) - 1, ptr)
    check_large(m, n, k, out, dtype, len(ptr) - 1, ptr, np.random.default_rng(n).permutation(n), seed=1)


def test_pointers_out_of_range_are_clamped(m):
    import torch
    rng = np.random.default_rng(10)
    q, e, w, we = random_operands(rng, 50, 64, 3, 32)
    a, b = rows_on_device(q, e), matrices_on_device(w, we)
    t = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        want = m.egnn_scaled_linear(*a, *b, ptr=t([0, 10, 20, 50]), dtype=dtype)
        assert torch.equal(m.egnn_scaled_linear(*a, *b, ptr=t([-5, 10, 20, 99]), dtype=dtype), want)
        perm = torch.arange(50, dtype=torch.int32, device="cuda")
        perm[49] = 1000
        assert torch.equal(m.egnn_scaled_linear(*a, *b, ptr=t([0, 10, 20, 50]), perm=perm, dtype=dtype), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k,out", [(9, 300, 300), (70, 700, 700), (300, 1030, 1030), (150, 64, 64)])
def test_every_code_counts(m, n, k, out, dtype):
    """One code in each row of W: every result is one exact product of 4 + 4 bits.  (fp16 has the small ones, down to 2^-9 2^-13 2^-4, rounded once.)"""
    import torch
    rng = np.random.default_rng(k)
    code, e, _ = R.quantise_rows(rng.standard_normal((n, k)) * 0.1)
    e[:] = rng.integers(-3, 4, e.shape)
    at = rng.permutation(k)[:out]
    w = np.zeros((1, out, k), np.uint8)
    w[0, np.arange(out), at] = rng.integers(0x30, 0x48, out)
    we = rng.integers(-3, 4, (1, -(-out // 128), -(-k // 128)))
    y = m.egnn_scaled_linear(*rows_on_device(code, e), *matrices_on_device(w, we), dtype=getattr(torch, dtype))
    want = R.values_of_rows(code, e) @ R.values_of_matrices(w, we)[0].T
    assert np.array_equal(values(y), want.astype(np.float16) if dtype == "float16" else want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k,out", [(5, 200, 40), (130, 200, 260), (40, 2000, 70), (300, 1500, 300)])
def test_sums_that_every_step_holds(m, n, k, out, dtype):
    """Codes of -1, 0 and 1, scaled by one block to the next: at most 100 of them count in a row of W."""
    import torch
    rng = np.random.default_rng(k)
    code = np.array([0x38, 0xB8], np.uint8)[rng.integers(0, 2, (n, k))]
    w = np.zeros((1, out, k), np.uint8)
    for r in range(out):
        w[0, r, rng.permutation(k)[:100]] = np.array([0x38, 0xB8], np.uint8)[rng.integers(0, 2, 100)]
    e = rng.integers(-9, 10, (n, 1)) * np.ones((1, -(-k // 128)), int)
    y = m.egnn_scaled_linear(*rows_on_device(code, e - 1), *matrices_on_device(w, np.ones((1, -(-out // 128), -(-k // 128)), int)), dtype=getattr(torch, dtype))
    assert np.array_equal(values(y), R.values_of_rows(code, e) @ R.values_of_matrices(w, np.zeros((1, -(-out // 128), -(-k // 128)), int))[0].T)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_scales_of_any_size(m, dtype):
    """Exponents whose sum is far inside the range though each is not."""
    import torch
    rng = np.random.default_rng(11)
    for ea, eb in ((-100, 95), (110, -105), (-127, 120), (60, 50), (-50, -50)):
        for n, k in ((5, 256), (200, 300)):
            q, e, w, we = random_operands(rng, n, k, 1, 90, 3)
            e, we = np.clip(e + ea, -127, 120), np.clip(we + eb, -127, 120)
            y = values(m.egnn_scaled_linear(*rows_on_device(q, e), *matrices_on_device(w, we), dtype=getattr(torch, dtype)))
            a, b = R.values_of_rows(q, e), R.values_of_matrices(w, we)[0]
            assert (np.abs(y - a @ b.T) <= bound(a @ b.T, np.abs(a) @ np.abs(b).T, k, dtype)).all()
    q, e, w, we = random_operands(rng, 20, 128, 1, 16)
    for ea, eb in ((-127, -127), (-100, -60)):
        y = m.egnn_scaled_linear(*rows_on_device(q, e * 0 + ea), *matrices_on_device(w, we * 0 + eb), dtype=getattr(torch, dtype))
        exact = R.values_of_rows(q, e * 0 + ea) @ R.values_of_matrices(w, we * 0 + eb)[0].T
        assert (np.abs(values(y) - exact) <= 2.0 ** -126).all()          # what is below the normal numbers may be zero
    y = m.egnn_scaled_linear(*rows_on_device(q, e * 0 + 120), *matrices_on_device(w, we * 0 + 120), dtype=getattr(torch, dtype))
    assert not torch.isfinite(y[values(y) != 0]).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_stays_in_its_row(m, dtype):
    import torch
    rng = np.random.default_rng(12)
    for n, k in ((7, 500), (150, 130)):
        q, e, w, we = random_operands(rng, n, k, 1, 70)
        want = m.egnn_scaled_linear(*rows_on_device(q, e), *matrices_on_device(w, we), dtype=getattr(torch, dtype))
        q[3, 100], w[0, 50, 7] = 0x7F, 0xFF
        y = m.egnn_scaled_linear(*rows_on_device(q, e), *matrices_on_device(w, we), dtype=getattr(torch, dtype))
        bad = torch.zeros_like(y, dtype=torch.bool)
        bad[3], bad[:, 50] = True, True
        assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], want[~bad])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift,wide", [(0, 130), (1, 131), (2, 140), (0, 256)])
def test_results_inside_a_larger_tensor(m, shift, wide, dtype):
    import torch
    rng = np.random.default_rng(13)
    for n, k in ((40, 128), (300, 64), (9, 1024)):
        q, e, w, we = random_operands(rng, n, k, 1, 120)
        a, b = rows_on_device(q, e), matrices_on_device(w, we)
        want = m.egnn_scaled_linear(*a, *b, dtype=getattr(torch, dtype))
        whole = torch.full((n * wide + shift,), 5.0, dtype=want.dtype, device="cuda")
        y = whole[shift:].view(n, wide)
        m.egnn_scaled_linear(*a, *b, y=y[:, :120])
        assert torch.equal(y[:, :120], want) and (y[:, 120:] == 5).all() and (whole[:shift] == 5).all()


def test_rows_of_codes_inside_wider_ones(m):
    """Codes of x and W in rows far longer than their codes, and rows of planes taken one after the other."""
    import torch
    rng = np.random.default_rng(14)
    q, e, w, we = random_operands(rng, 60, 80, 1, 50)
    a, b = rows_on_device(q, e), matrices_on_device(w, we)
    want = m.egnn_scaled_linear(*a, *b)
    far = torch.full((60, 240), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    far[:, :80] = a[0]
    wfar = torch.full((1, 50, 144), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    wfar[:, :, :80] = b[0]
    assert torch.equal(m.egnn_scaled_linear(far[:, :80], a[1], wfar[:, :, :80], b[1]), want)
    assert torch.equal(m.egnn_scaled_linear(a[0].view(12, 5, 80), a[1].view(12, 5, 1), *b), want)


def test_codes_past_32_bits(m):
    """Rows of codes 100,000 bytes apart and rows of y 60,000 values apart, the last ones behind 2^32 of them."""
    import torch
    rng = np.random.default_rng(15)
    n = 80000
    x = torch.randn(n, 32, device="cuda")
    a = m.egnn_quantise_rows(x)
    b = m.egnn_quantise_matrices(torch.randn(1, 16, 32, device="cuda"))[:2]
    want = m.egnn_scaled_linear(*a, *b, dtype=torch.bfloat16)
    far = torch.empty((n, 100000 // 16 * 16), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    far[:, :32] = a[0]
    y = torch.empty((n, 60000), dtype=torch.bfloat16, device="cuda")
    m.egnn_scaled_linear(far[:, :32], a[1], *b, y=y[:, :16])
    assert torch.equal(y[:, :16], want)


def test_no_rows(m):
    import torch
    b = m.egnn_quantise_matrices(torch.randn(2, 16, 32, device="cuda"))[:2]
    a = m.egnn_quantise_rows(torch.empty(0, 32, device="cuda"))
    assert m.egnn_scaled_linear(*a, *b, ptr=torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 16)


def test_captured_and_the_same_every_time(m):
    import torch
    rng = np.random.default_rng(16)
    for n, k, out in ((3, 4096, 64), (500, 64, 64), (400, 512, 300)):
        x, W = torch.randn(n, k, device="cuda"), torch.randn(2, out, k, device="cuda")
        ptr = torch.tensor([0, n // 3, n], dtype=torch.int32, device="cuda")
        for dtype in (torch.float32, torch.bfloat16):
            a, b = m.egnn_quantise_rows(x), m.egnn_quantise_matrices(W)[:2]
            y = m.egnn_scaled_linear(*a, *b, ptr=ptr, dtype=dtype)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                m.egnn_quantise_rows(x, *a)
                m.egnn_scaled_linear(*a, *b, ptr=ptr, y=y)
            for _ in range(3):
                x.mul_(1.3)
                want = m.egnn_scaled_linear(*m.egnn_quantise_rows(x), *b, ptr=ptr, dtype=dtype)
                y.zero_()
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k,out,groups", [(1, 1, 8, 1), (9, 100, 40, 1), (300, 20, 33, 1), (500, 50, 64, 3), (700, 100, 17, 2), (70, 90, 64, 1), (20, 130, 70, 1),
                                            (5, 2049, 48, 1), (130, 1001, 200, 1), (900, 200, 300, 4), (1300, 650, 520, 1), (3600, 2057, 3400, 1), (5120, 140, 5000, 1),
                                            (3600, 2177, 3400, 1)])
def test_columns_of_wider_codes(m, n, k, out, groups, dtype):
    """Bytes behind the last code of a row, up to a multiple of 16, are not part of it: codes taken out of wider ones, and NaN there."""
    import torch
    torch.manual_seed(k)
    wide = (k + 15) // 16 * 16 + 16
    ptr = None if groups == 1 else torch.tensor([0] + [n * (g + 1) // groups for g in range(groups)], dtype=torch.int32, device="cuda")
    a, b = m.egnn_quantise_rows(torch.randn(n, k, device="cuda")), m.egnn_quantise_matrices(torch.randn(groups, out, k, device="cuda"))[:2]
    want = m.egnn_scaled_linear(*a, *b, ptr=ptr, dtype=getattr(torch, dtype))
    for qfill, wfill in ((0x7F, 0x7F), (0x38, 0x38), (0xFF, 0x01)):
        q = torch.full((n, wide), qfill, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        w = torch.full((groups, out, wide), wfill, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        q[:, :k], w[:, :, :k] = a[0], b[0]
        assert torch.equal(m.egnn_scaled_linear(q[:, :k], a[1], w[:, :, :k], b[1], ptr=ptr, dtype=getattr(torch, dtype)), want)
