"""The trained block (species_block.py): its gradients against the fp64 oracle's chain and against differences, its equivariance, and
that training it goes down."""
import numpy as np
import pytest

from oracle import block_oracle as K

pytestmark = pytest.mark.gpu


def make(lmax=2, channels=16, n=50, ptr=None):
    import torch
    from paper_2507_03840_amd import binding as B
    from paper_2507_03840_amd.species_block import SpeciesBlock
    rng = np.random.default_rng([11, lmax, channels])
    lib = B.Egnn(lmax, channels, 8, 5.0, 10.0)
    species = rng.integers(0, 3, n).astype(np.int32)
    p = None if ptr is None else torch.tensor(ptr, dtype=torch.int32, device="cuda")
    block = SpeciesBlock(lib, torch.from_numpy(species).cuda(), 3, ptr=p)
    block.bias += torch.randn_like(block.bias) * block.degree0
    block.gamma += 0.1 * torch.randn_like(block.gamma)
    block.beta += 0.1 * torch.randn_like(block.beta)
    x = torch.randn((n, lib.dim, channels), device="cuda")
    return lib, block, species, x


def oracle_forward(lib, species, x, W, bias, gamma, beta, ptr):
    n, dim, c = x.shape
    h = x.copy()
    h[:, 0] = K.group_norm(x[:, 0], 4, gamma, beta, ptr)[0]
    row_ptr, perm = K.group_rows(species, 3, lib.lmax)
    return x + K.grouped_linear(h.reshape(n * dim, c), W, row_ptr, perm, bias)[0].reshape(x.shape)


@pytest.mark.parametrize("lmax,channels,ptr", [(0, 8, None), (2, 16, None), (4, 32, [0, 20, 20, 50])])
def test_forward_and_gradients(lmax, channels, ptr):
    """fp32 against fp64 (relative to the largest value, 2e-5 as in the other chains of this suite), and central differences of the oracle."""
    import torch
    lib, block, species, x = make(lmax, channels, ptr=ptr)
    f = lambda t: t.double().cpu().numpy()
    names = ("W", "bias", "gamma", "beta")
    w = {k: f(getattr(block, k)) for k in names}
    out = block.forward(x)
    ref = oracle_forward(lib, species, f(x), *(w[k] for k in names), ptr)
    assert np.abs(f(out) - ref).max() <= 2e-5 * np.abs(ref).max()
    dout = torch.randn_like(out)
    dx, grads = block.backward(dout)
    rng = np.random.default_rng(5)
    for name, value, grad in [("x", f(x), f(dx))] + [(k, w[k], f(grads[k])) for k in names]:
        d = rng.standard_normal(value.shape)
        if name == "bias":
            d = d * f(block.degree0)
        at = lambda s: (oracle_forward(lib, species, value + s * d if name == "x" else f(x), *(value + s * d if k == name else w[k] for k in names), ptr) * f(dout)).sum()
        want, got = (at(1e-5) - at(-1e-5)) / 2e-5, (grad * d).sum()
        assert abs(want - got) <= 1e-5 * np.abs(grad * d).sum() + 1e-6, name


def test_equivariant():
    """A rotation of every degree's components commutes with the block: here the signs of x and y (half a turn about z)."""
    import torch
    lib, block, _, x = make(3, 16)
    sign = torch.tensor([(-1.0) ** abs(m) for l in range(4) for m in range(-l, l + 1)], device="cuda")[None, :, None]
    assert (block.forward(x * sign) - block.forward(x) * sign).abs().max() <= 1e-5


def test_training_goes_down():
    from paper_2507_03840_amd.species_block import train
    losses = train(verbose=False)
    assert losses[-1] < 0.1 * losses[0], (losses[0], losses[-1])
