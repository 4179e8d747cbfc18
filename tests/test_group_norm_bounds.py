"""The bounds of tests/group_norm_bounds.py hold the fp32 formula and tell it from one with a term or a few rows left out (no GPU needed)."""
import numpy as np
import pytest

from oracle import block_oracle as K
from tests.group_norm_bounds import CASES, HALF_STEP, adjoint, inputs

STEP = {"float32": 23, "float16": 10, "bfloat16": 7}


def rounded(a, dtype):
    m, e = np.frexp(a)
    return np.ldexp(np.round(np.ldexp(m, STEP[dtype] + 1)), e - STEP[dtype] - 1)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%dx%d" % c[:2])
def test_bounds(case, dtype):
    x, dy, gamma, beta = inputs(case)
    x, dy = rounded(x, dtype), rounded(dy, dtype)
    n, c, groups, ptr = case[:4]
    dx, bound, (own, mean, along) = adjoint(case, x, dy, gamma, beta, dtype)
    assert np.allclose(dx, K.group_norm_backward(x, dy, groups, gamma, beta, ptr)[0], rtol=1e-9, atol=1e-12)
    assert (np.abs(rounded(dx, dtype) - dx) <= bound).all()
    # each term by itself, where a group has more than one value
    short = ptr is not None and min(b - a for a, b in zip(ptr[:-1], ptr[1:]) if b > a) * (c // groups) < 3
    if n * (c // groups) > 4 and not short:
        for wrong in (own - along, own - mean, own, 0 * own):
            assert (np.abs(rounded(wrong, dtype) - dx) > bound).any()
    # the means without the last 64 rows of the longest segment
    at = [0, n] if ptr is None else ptr
    b, e = max(zip(at[:-1], at[1:]), key=lambda p: p[1] - p[0])
    if e - b > 200:
        lost = own.copy()
        for t, f in ((mean, 1.0), (along, None)):
            size = c // groups
            _, mu, r = K.group_norm(x, groups, gamma, beta, ptr)
            s = next(i for i, p in enumerate(zip(at[:-1], at[1:])) if p == (b, e))
            h = (x[b:e] - np.repeat(mu[s], size)) * np.repeat(r[s], size)
            v = own[b:e] * (1.0 if f else h)
            m = np.repeat(v[:-64].reshape(e - b - 64, groups, size).sum((0, 2)) / ((e - b) * size), size)
            lost[b:e] -= m * (1.0 if f else h)
        assert (np.abs(rounded(lost, dtype)[b:e] - dx[b:e]) > bound[b:e]).any()
