"""How near orthogonalised updates come to oracle/block_oracle.py (fp64): bounds that the loss of a piece of an operand would break."""
import numpy as np
import pytest

from oracle import block_oracle as K

pytestmark = pytest.mark.gpu
FULL = 5 * 8 * 10.25 * 2.0 ** -24      # five steps, 8 roundings of each of their terms (a + |b| + |c| = 10.25 parts of x)


@pytest.fixture(scope="module")
def m():
    from paper_2507_03840_amd import binding as B
    return B.Egnn(2, 32, 16, 10.0, 200.0)


def random(rng, *shape):
    """A few strong directions over many weak ones, as gradients have."""
    b, n, m = shape
    r = max(1, min(n, m) // 8)
    return 1e-3 * (rng.standard_normal(shape) + 2.0 * rng.standard_normal((b, n, r)) @ rng.standard_normal((b, r, m)))


@pytest.mark.parametrize("dtype,bits,least", [("bfloat16", 8, 0.0), ("float16", 11, 2.0 ** -25)])
@pytest.mark.parametrize("shape", [(2, 20, 30), (1, 64, 300), (2, 100, 90), (1, 300, 301), (2, 320, 480), (1, 256, 1000), (1, 1300, 400)])
def test_fewer_bits_are_the_last_rounding_alone(m, shape, dtype, bits, least):
    """v before the rounding is off by FULL in the 2-norm.  y, v rounded to nearest, is off by at most half a step at the exact value and twice
    what v is off (where v lies across a power of two, the half step there is wider, but the power itself is no farther from v than
    the exact value is)."""
    import torch
    g = torch.from_numpy(random(np.random.default_rng([1, *shape]), *shape)).to(getattr(torch, dtype)).cuda()
    want = K.orthogonalise(g.double().cpu().numpy())
    half = np.maximum(np.ldexp(1.0, np.frexp(want)[1] - 1 - bits), least)
    beyond = np.maximum(np.abs(m.egnn_orthogonalise(g).double().cpu().numpy() - want) - half, 0.0)
    print(shape, dtype, "beyond half a step: %.2e" % (np.linalg.norm(beyond) / np.linalg.norm(want)))
    assert np.linalg.norm(beyond) <= 2 * FULL * np.linalg.norm(want)
