"""A trained block between two layers, made of the library's calls: SiLU group norm of the scalar channels, a linear map per (species,
degree) of every row, a residual connection, and orthogonalised updates of the maps.

    python -m paper_2507_03840_amd.species_block          # trains one on the 64-atom cluster towards a fixed random block

The norm sees the degree-0 plane alone, per structure; maps mix channels and never the components m of a degree, and only degree 0 has a
bias: the block is equivariant under rotations, as the layers on both sides of it are."""
import torch

from . import binding as B


class SpeciesBlock:
    """Weights and the buffers kept from step to step for nodes [n][(lmax + 1)^2][channels]."""

    def __init__(self, lib, species, n_species, groups=4, ptr=None, seed=0):
        self.lib, self.groups, self.ptr, self.n_species = lib, groups, ptr, n_species
        c, degrees = lib.channels, lib.lmax + 1
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.W = torch.randn((n_species * degrees, c, c), generator=gen, device="cuda") * c ** -0.5
        self.bias = torch.zeros((n_species * degrees, c), device="cuda")
        self.gamma, self.beta = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
        self.momentum = torch.zeros_like(self.W)
        self.degree0 = (torch.arange(n_species * degrees, device="cuda") % degrees == 0).float()[:, None]
        n = species.numel()
        self.row_ptr, self.perm = lib.egnn_group_rows(species, n_species, lmax=lib.lmax)      # species do not change between steps
        segments = 1 if ptr is None else ptr.numel() - 1
        nbytes = max(lib.egnn_group_norm_workspace_bytes(n, segments, c, groups),
                     lib.egnn_grouped_linear_workspace_bytes(n * lib.dim, n_species * degrees, c, c),
                     lib.egnn_orthogonalise_workspace_bytes(n_species * degrees, c, c))
        self.ws = torch.empty(max(256, nbytes), dtype=torch.uint8, device="cuda")

    def forward(self, x):
        """x [n][(lmax + 1)^2][channels] -> the same shape; keeps what the adjoint needs."""
        n, dim, c = x.shape
        self.x, self.h = x, x.clone()
        _, self.mean, self.rstd = self.lib.egnn_group_norm(x[:, 0], self.groups, self.gamma, self.beta, ptr=self.ptr, y=self.h[:, 0],
                                                           ws=self.ws)
        y = self.lib.egnn_grouped_linear(self.h.view(n * dim, c), self.W, self.row_ptr, perm=self.perm, bias=self.bias)
        return x + y.view(n, dim, c)

    def backward(self, dout):
        """(dx, gradients of the weights by name)."""
        n, dim, c = dout.shape
        dh, dW, db = self.lib.egnn_grouped_linear_backward(self.h.view(n * dim, c), self.W, dout.reshape(n * dim, c), self.row_ptr,
                                                           perm=self.perm, ws=self.ws)
        dh = dh.view(n, dim, c)
        _, dgamma, dbeta = self.lib.egnn_group_norm_backward(self.x[:, 0], dh[:, 0], self.mean, self.rstd, self.groups, self.gamma,
                                                             self.beta, ptr=self.ptr, dx=dh[:, 0], ws=self.ws)
        return dout + dh, dict(W=dW, bias=db * self.degree0, gamma=dgamma, beta=dbeta)

    def step(self, grads, lr):
        """Maps by orthogonalised updates, vectors along their gradients."""
        self.lib.egnn_muon_step(self.W, grads["W"], self.momentum, lr, ws=self.ws)
        for name in ("bias", "gamma", "beta"):
            getattr(self, name).sub_(grads[name], alpha=lr)


def train(steps=60, lr=0.1, verbose=True):
    """Mean squared distance from a fixed random block on the 64-atom cluster, before every step."""
    from . import synth
    w = synth.workload(1)
    lib = B.Egnn(w.lmax, w.channels, w.n_rbf, w.r_cut, 10.0, orb_l=w.orb_l)
    species = B.to_device(w.species).to(torch.int32)
    n_species = int(species.max()) + 1
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn((species.numel(), lib.dim, lib.channels), generator=gen, device="cuda")
    target = SpeciesBlock(lib, species, n_species, seed=2).forward(x)
    block, losses = SpeciesBlock(lib, species, n_species, seed=3), []
    for k in range(steps):
        off = block.forward(x) - target
        losses.append(off.square().mean())
        _, grads = block.backward(off * (2.0 / off.numel()))
        block.step(grads, lr * (1.0 - k / steps))
    losses = [float(v) for v in losses]
    if verbose:
        print("loss " + " ".join(f"{v:.4f}" for v in losses[:: max(1, steps // 8)]) + f" ... {losses[-1]:.4f}")
    return losses


if __name__ == "__main__":
    train()
