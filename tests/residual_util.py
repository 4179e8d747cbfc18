"""Tensors and bounds that the tests of the residual block's calls share."""
import numpy as np

from oracle import residual_oracle as R

U32 = 2.0 ** -24
HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
FLOOR = {"float32": 2.0 ** -150, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -134}   # half a step of the smallest numbers


def values(t):
    return t.double().cpu().numpy()


def codes(q):
    """Bytes of a tensor of codes."""
    import torch
    return q.contiguous().view(torch.uint8).cpu().numpy()


def exponents(scale):
    import torch
    return scale.view(torch.uint8).cpu().numpy().astype(np.int64) - 127


def padding(q):
    """The bytes between the last code of each row and the next multiple of 16."""
    import torch
    n = q.shape[-1]
    whole = q.as_strided((*q.shape[:-1], (n + 15) // 16 * 16), q.stride())
    return whole.contiguous().view(torch.uint8)[..., n:].cpu().numpy()


def check_codes(q, scale, y, error=0.0):
    """Codes and scales of rows y [n][cols] (fp64) that the kernel knew up to error * |y|: each code is within half a step of its value."""
    want, e, on = R.quantise_rows(y)
    got = exponents(scale).reshape(e.shape)
    code = codes(q).reshape(want.shape)
    if error == 0.0:
        assert np.array_equal(got, e) and np.array_equal(code, want)
        return
    blocks = np.array([[np.abs(y[r, b * 128:(b + 1) * 128]).max() for b in range(e.shape[1])] for r in range(len(y))]).reshape(e.shape)
    beside = np.abs(blocks / (448.0 * 2.0 ** np.minimum(got, e).astype(float)) - 1) <= error       # a largest value next to where the scale changes
    assert ((got == e) | (beside & (np.abs(got - e) == 1))).all()
    on = y * np.repeat(2.0 ** -got.astype(float), 128, 1)[:, :y.shape[1]]
    size = np.maximum(np.abs(on), 2.0 ** -6)
    half = 2.0 ** (np.floor(np.log2(size)) - 4)
    assert (np.abs(R.decode(code) - on) <= half * (1 + 1e-12) + error * np.abs(on)).all()


def check_gradients(case, dx, dgamma, dW, off=0.0):
    """Gradients of a block y = norm(h) gamma, z = W y by group, with the loss sum(z d) + sum(h dh), against differences of it in fp64.

    case: h, gamma, W, d, dh (fp64), ptr, perm, and the values W8 and d8 that the codes of W and d stand for.
    1. With the roundings to 8 bits held: dx and dgamma are those of sum(norm(h) gamma W8 d8) + sum(h dh), dW that of sum(z d).  Directions of random signs;
       the difference is that of the gradients' own error, `off` of the sum of magnitudes of their terms, and 1e-7 of the sum of |g u| for the central
       differences (step 1e-4 of values around 1: a third derivative of a few times the first one, / 6, times 1e-8).
    2. Without them: along the gradient g itself, whose terms do not cancel, g . g.  A product of two codes is within (1 + 2^-4)^2 - 1 of that of the
       values, up or down by chance, so that along g no more than that part of g . g is missing."""
    from oracle import block_oracle as K
    h, gamma, W, d, dh, ptr, perm, W8, d8 = (case[k] for k in ("h", "gamma", "W", "d", "dh", "ptr", "perm", "W8", "d8"))
    n, dim, c = h.shape
    rng, t = np.random.default_rng(len(h)), 1e-4

    def loss(h, gamma, W, d):
        z, _ = K.grouped_linear(R.rms_norm(h, gamma).reshape(n * dim, c), W, ptr, perm)
        return (z * d).sum() + (h * dh).sum()

    def along(W, d, a=0.0, b=0.0, e=0.0):
        return (loss(h + t * a, gamma + t * b, W + t * e, d) - loss(h - t * a, gamma - t * b, W - t * e, d)) / (2 * t)

    dy8, dsize = K.grouped_linear(d8, W8.transpose(0, 2, 1), ptr, perm)
    _, _, xterms, gterms = R.rms_norm_backward(h, dy8.reshape(h.shape), gamma, dh)
    _, _, xthrough, gthrough = R.rms_norm_backward(h, dsize.reshape(h.shape), gamma)
    _, _, _, _, wterms, _ = K.grouped_linear_backward(R.rms_norm(h, gamma).reshape(n * dim, c), W, d, ptr, perm)
    for _ in range(4):
        a, b, e = (rng.choice([-1.0, 1.0], v.shape) for v in (h, gamma, W))
        for got, terms, want in ((dx * a, xterms + xthrough, along(W8, d8, a=a)), (dgamma * b, gterms + gthrough, along(W8, d8, b=b)), (dW * e, wterms, along(W, d, e=e))):
            assert abs(got.sum() - want) <= off * terms.sum() + 1e-7 * np.abs(got).sum()
    dy, _ = K.grouped_linear(d, W.transpose(0, 2, 1), ptr, perm)
    gx, gg, _, _ = R.rms_norm_backward(h, dy.reshape(h.shape), gamma, dh)
    _, gW, _, _, _, _ = K.grouped_linear_backward(R.rms_norm(h, gamma).reshape(n * dim, c), W, d, ptr, perm)
    for got, g, want in ((dx, gx, along(W, d, a=gx)), (dgamma, gg, along(W, d, b=gg)), (dW, gW, along(W, d, e=gW))):
        assert abs((g * g).sum() - want) <= 1e-6 * (g * g).sum()
        assert abs((got * g).sum() - want) <= ((1 + 2.0 ** -4) ** 2 - 1) * want


def block_case(rng, lmax, channels, n, n_species):
    """Inputs of check_gradients of a block with nodes of n atoms, in fp64, and the oracle's gradients at them with its own codes."""
    from oracle import block_oracle as K
    dim = (lmax + 1) ** 2
    ptr, perm = K.group_rows(rng.integers(0, n_species, n), n_species, lmax)
    h, dh = rng.standard_normal((2, n, dim, channels))
    gamma = 1 + 0.2 * rng.standard_normal((lmax + 1, channels))
    W, d = rng.standard_normal((n_species * (lmax + 1), channels, channels)) * channels ** -0.5, rng.standard_normal((n * dim, channels))
    case = dict(h=h, gamma=gamma, W=W, d=d, dh=dh, ptr=ptr, perm=perm, W8=R.values_of_matrices(*R.quantise_matrices(W)), d8=R.values_of_rows(*R.quantise_rows(d)[:2]))
    dy, _ = K.grouped_linear(case["d8"], case["W8"].transpose(0, 2, 1), ptr, perm)
    dx, dgamma, _, _ = R.rms_norm_backward(h, dy.reshape(h.shape), gamma, dh)
    _, dW, _, _, _, _ = K.grouped_linear_backward(R.rms_norm(h, gamma).reshape(n * dim, channels), W, d, ptr, perm)
    return case, dx, dgamma, dW, dy.reshape(h.shape)
