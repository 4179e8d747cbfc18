"""The group norm and its adjoint against fp64 (oracle/block_oracle.py and formulas), with bounds that follow each value."""
import numpy as np
import pytest

from oracle import block_oracle as K
from tests.group_norm_bounds import CASES, adjoint, forward, inputs

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def m():
    from paper_2507_03840_amd import binding as B
    return B.Egnn(2, 32, 16, 10.0, 200.0)


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("n,c,segments", [(150000, 701, 1), (30000, 64, 3000), (30000, 1000, 3000)])
def test_sums_of_equal_terms(m, n, c, segments, dtype):
    """Equal rows: xhat = 0, z = beta, every term of dbeta is dy SiLU'(beta), and each fp32 addition of it would be rounded to the same side.
    A term is off by 12 roundings of (1 + |beta|) |dy|, the sum by 4 additions in fp32, 9 levels of a tree and 3 roundings between them."""
    import torch
    t = getattr(torch, dtype)
    beta = np.random.default_rng([1, c]).uniform(-2, 2, c).astype(np.float32)
    b = torch.from_numpy(beta).cuda()
    one = torch.ones(c, device="cuda")
    x, dy = torch.full((n, c), 0.75, dtype=t, device="cuda"), torch.full((n, c), 0.7, dtype=t, device="cuda")
    ptr = None if segments == 1 else torch.arange(0, n + 1, n // segments, dtype=torch.int32, device="cuda")
    _, mean, rstd = m.egnn_group_norm(x, 1, one, b, ptr=ptr)
    assert (mean == 0.75).all()
    _, dgamma, dbeta = m.egnn_group_norm_backward(x, dy, mean, rstd, 1, one, b, ptr=ptr)
    sig = K.sigmoid(beta.astype(np.float64))
    d = float(dy[0, 0])
    want = n * d * sig * (1 + beta * (1 - sig))
    off = np.abs(dbeta.double().cpu().numpy() - want)
    print("off by at most %.1f of 2^-24 of n |dy|" % (off.max() / (U32 * n * d)))
    assert (off <= U32 * n * d * (12 * (1 + np.abs(beta)) + 16 * 1.1)).all()
    assert not dgamma.any()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%dx%d" % c[:2])
def test_every_value_within_its_own_bound(m, case, dtype):
    """y and dx against fp64 with bounds that a missing term or a few missing rows break (test_group_norm_bounds.py shows that they do)."""
    import torch
    t = getattr(torch, dtype)
    n, c, groups, ptr = case[:4]
    x, dy, gamma, beta = inputs(case)
    x, dy = (torch.from_numpy(a).to(t).cuda() for a in (x, dy))
    g, b = torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
    p = None if ptr is None else torch.tensor(ptr, dtype=torch.int32, device="cuda")
    at = lambda a: a.double().cpu().numpy()
    y, mean, rstd = m.egnn_group_norm(x, groups, g, b, ptr=p)
    want, bound = forward(case, at(x), gamma, beta, dtype)
    print("y: %.2f of the bound" % (np.abs(at(y) - want) / bound).max())
    assert (np.abs(at(y) - want) <= bound).all()
    dx, _, _ = m.egnn_group_norm_backward(x, dy, mean, rstd, groups, g, b, ptr=p)
    want, bound, _ = adjoint(case, at(x), at(dy), gamma, beta, dtype)
    print("dx: %.2f of the bound" % (np.abs(at(dx) - want) / bound).max())
    assert (np.abs(at(dx) - want) <= bound).all()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("n,c", [(1, 96), (1, 7), (2, 96), (5, 33), (300, 64), (4000, 20)])
def test_groups_of_one_value_have_no_gradient(m, n, c, dtype):
    """A group of one value is its own mean: xhat = 0 and dx = rstd (gamma dz - gamma dz), with rstd = 316.  What the mean of one term is rounded
    to would be all of the result, and is most of it in groups of two."""
    import torch
    rng = np.random.default_rng([6, n, c])
    t = getattr(torch, dtype)
    x, dy = (torch.from_numpy(rng.standard_normal((n, c))).to(t).cuda() for _ in range(2))
    g, b = (torch.from_numpy(rng.standard_normal(c)).float().cuda() for _ in range(2))
    ptr = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    _, mean, rstd = m.egnn_group_norm(x, c, g, b, ptr=ptr)
    assert torch.equal(mean, x.float())
    dx, _, dbeta = m.egnn_group_norm_backward(x, dy, mean, rstd, c, g, b, ptr=ptr)
    assert not dx.any() and dbeta.all()
