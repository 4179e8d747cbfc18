"""The adjoint of the group norm against fp64 (oracle/block_oracle.py and formulas), with bounds that follow each value."""
import numpy as np
import pytest

from oracle import block_oracle as K

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
