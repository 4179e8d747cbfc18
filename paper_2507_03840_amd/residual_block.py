"""Residual blocks whose products are in 8 bits, made of the library's calls: the sum with what the block before gave, its root-mean-square norm by
degree, a linear map per (species, degree) of every row, and steps of limited, orthogonalised updates.

    python -m paper_2507_03840_amd.residual_block         # trains a stack on the 64-atom cluster towards a fixed random one

    h_k = x_k + h_(k-1),  x_(k+1) = W (norm of h_k)        (h_(-1) = 0; the stack's result is x + h of the last block)

Norm and maps mix no components m of a degree, and only degree 0 has a bias: up to the rounding to 8 bits a stack is equivariant under rotations.  The
weights are kept in fp32; their codes, in both orders, are made again after every step.  On the way back the gradient of a map's result is
rounded to 8 bits for the product with the transposed codes; weights get theirs from the rows as they are."""
import torch

from . import binding as B


class ResidualBlock:
    """Weights and the buffers kept from step to step for nodes [n][(lmax + 1)^2][channels] in fp32."""

    def __init__(self, lib, species, n_species, seed=0):
        self.lib = lib
        c, degrees = lib.channels, lib.lmax + 1
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.W = torch.randn((n_species * degrees, c, c), generator=gen, device="cuda") * c ** -0.5
        self.bias = torch.zeros((n_species * degrees, c), device="cuda")
        self.gamma = torch.ones((degrees, c), device="cuda")
        self.momentum = torch.zeros_like(self.W)
        self.degree0 = (torch.arange(n_species * degrees, device="cuda") % degrees == 0).float()[:, None]
        n = species.numel()
        self.ptr, self.perm = lib.egnn_group_rows(species, n_species, lmax=lib.lmax)      # species do not change between steps
        self.room = torch.empty(max(256, lib.egnn_rms_norm_workspace_bytes(n, lib.lmax, c),
                                    lib.egnn_grouped_linear_workspace_bytes(n * lib.dim, n_species * degrees, c, c),
                                    lib.egnn_orthogonalise_workspace_bytes(n_species * degrees, c, c)), dtype=torch.uint8, device="cuda")
        self.code = lib.egnn_quantise_matrices(self.W, qt=None)
        self.h = self.y = None                      # of the last forward pass that was kept

    def forward(self, x, h=None, keep=True):
        """(x, sum so far) [n][(lmax + 1)^2][channels] -> (the next block's x, h); keep: what the adjoint needs (else what an earlier pass kept goes too)."""
        n, dim, c = x.shape
        y, h, q, scale = self.lib.egnn_rms_norm(x, self.gamma, residual=h, y=None if keep else False, q=None)
        out = self.lib.egnn_scaled_linear(q, scale, *self.code[:2], ptr=self.ptr, perm=self.perm, bias=self.bias)
        self.h, self.y = (h, y) if keep else (None, None)
        return out.view(n, dim, c), h

    def backward(self, dout, dh=None):
        """Gradients of the last forward pass's results -> (gradient of x, which is also that of the sum so far, gradients of the weights by name)."""
        if self.h is None:
            raise RuntimeError("backward: the last forward pass kept nothing, or there was none")
        n, dim, c = dout.shape
        rows = dout.reshape(n * dim, c)
        dy = self.lib.egnn_scaled_linear(*self.lib.egnn_quantise_rows(rows), *self.code[2:], ptr=self.ptr, perm=self.perm)
        _, dW, db = self.lib.egnn_grouped_linear_backward(self.y.view(n * dim, c), self.W, rows, self.ptr, perm=self.perm, dx=False, ws=self.room)
        dx, dgamma = self.lib.egnn_rms_norm_backward(self.h, dy.view(n, dim, c), self.gamma, dh=dh, ws=self.room)
        return dx, dict(W=dW, bias=db * self.degree0, gamma=dgamma)

    def step(self, grads, lr):
        """Maps by orthogonalised updates, vectors along their gradients; then the maps' codes."""
        self.lib.egnn_muon_step(self.W, grads["W"], self.momentum, lr, ws=self.room)
        for name in ("bias", "gamma"):
            getattr(self, name).sub_(grads[name], alpha=lr)
        self.lib.egnn_quantise_matrices(self.W, *self.code)


class ResidualStack:
    def __init__(self, lib, species, n_species, depth, seed=0):
        self.lib = lib
        self.blocks = [ResidualBlock(lib, species, n_species, seed=1000 * seed + k) for k in range(depth)]

    def forward(self, x, keep=True):
        h = None
        for block in self.blocks:
            x, h = block.forward(x, h, keep)
        return x + h

    def backward(self, dout):
        """Gradient of the stack's result -> (gradient of its input, gradients of the blocks)."""
        dx, dh, grads = dout, dout, []
        for block in reversed(self.blocks):
            dx, g = block.backward(dx, dh)
            dh = dx
            grads.append(g)
        return dx, grads[::-1]

    def step(self, grads, lr, max_norm=1.0):
        """One step with the gradients' common norm limited; returns that norm.  Nothing is changed where it is not finite."""
        norm, factor = self.lib.egnn_clip_gradients([g[name] for g in grads for name in ("W", "bias", "gamma")], max_norm).tolist()
        if factor > 0.0:
            for block, g in zip(self.blocks, grads):
                block.step(g, lr)
        return norm


def train(steps=40, lr=0.05, depth=3, verbose=True):
    """Mean squared distance from a fixed random stack on the 64-atom cluster, before every step, and the gradients' norms."""
    from . import synth
    w = synth.workload(1)
    lib = B.Egnn(w.lmax, w.channels, w.n_rbf, w.r_cut, 10.0, orb_l=w.orb_l)
    species = B.to_device(w.species).to(torch.int32)
    n_species = int(species.max()) + 1
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn((species.numel(), lib.dim, lib.channels), generator=gen, device="cuda")
    target = ResidualStack(lib, species, n_species, depth, seed=2).forward(x, keep=False)
    stack, losses, norms = ResidualStack(lib, species, n_species, depth, seed=3), [], []
    for k in range(steps):
        off = stack.forward(x) - target
        losses.append(off.square().mean())
        _, grads = stack.backward(off * (2.0 / off.numel()))
        norms.append(stack.step(grads, lr * (1.0 - k / steps)))
    losses = [float(v) for v in losses]
    if verbose:
        print("loss " + " ".join(f"{v:.4f}" for v in losses[:: max(1, steps // 8)]) + f" ... {losses[-1]:.4f}, gradient norm {norms[0]:.3f} ... {norms[-1]:.3f}")
    return losses, norms


if __name__ == "__main__":
    train()
