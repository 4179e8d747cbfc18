"""fp64 oracle of a residual block in 8 bits: root-mean-square norm by degree, codes with scales, products of codes, clipping.  Plain
numpy from the formulas; no code shared with the library."""
import numpy as np

BLOCK = 128
# the 127 finite magnitudes of e4m3, by code: subnormals m 2^-9, then (8 + m) 2^(e - 10)
MAGNITUDES = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def decode(code):
    """Values of e4m3 codes (uint8)."""
    code = np.asarray(code, np.uint8)
    v = np.append(MAGNITUDES, np.nan)[code & 0x7F]
    return np.where(code & 0x80, -v, v)


def encode(v):
    """Codes nearest to values of magnitude at most 448, ties to the even code; NaN for what is not finite."""
    v = np.asarray(v, np.float64)
    a = np.where(np.isfinite(v), np.abs(v), 0.0)
    assert (a <= 448).all()
    hi = np.clip(np.searchsorted(MAGNITUDES, a), 0, 126)          # first magnitude >= a
    lo = np.maximum(hi - 1, 0)
    up, down = MAGNITUDES[hi] - a, a - MAGNITUDES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isfinite(v), code, 0x7F)
    return (code | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def exponent(largest):
    """The least integer e >= -127 with largest <= 448 * 2^e."""
    e = -127
    if largest > 0:
        e = max(e, int(np.floor(np.log2(largest))) - 10)
        while largest > 448.0 * 2.0 ** e:
            e += 1
    return e


def _largest(v):
    return np.abs(np.where(np.isfinite(v), v, 0.0)).max(initial=0.0)


def quantise_rows(x):
    """(codes, exponents, values on their scale) of rows [n][cols]."""
    x = np.asarray(x, np.float64)
    n, cols = x.shape
    q, e, on = np.zeros(x.shape, np.uint8), np.zeros((n, -(-cols // BLOCK)), np.int64), np.zeros(x.shape)
    for r in range(n):
        for b in range(e.shape[1]):
            at = slice(b * BLOCK, (b + 1) * BLOCK)
            e[r, b] = exponent(_largest(x[r, at]))
            on[r, at] = x[r, at] * 2.0 ** -float(e[r, b])
            q[r, at] = encode(on[r, at])
    return q, e, on


def quantise_matrices(W):
    W = np.asarray(W, np.float64)
    batch, rows, cols = W.shape
    q, e = np.zeros(W.shape, np.uint8), np.zeros((batch, -(-rows // BLOCK), -(-cols // BLOCK)), np.int64)
    for b in range(batch):
        for i in range(e.shape[1]):
            for j in range(e.shape[2]):
                at = (b, slice(i * BLOCK, (i + 1) * BLOCK), slice(j * BLOCK, (j + 1) * BLOCK))
                e[b, i, j] = exponent(_largest(W[at]))
                q[at] = encode(W[at] * 2.0 ** -float(e[b, i, j]))
    return q, e


def values_of_rows(q, e):
    return decode(q) * np.repeat(2.0 ** e.astype(np.float64), BLOCK, 1)[:, :q.shape[1]]


def values_of_matrices(q, e):
    s = np.repeat(np.repeat(2.0 ** e.astype(np.float64), BLOCK, 1), BLOCK, 2)
    return decode(q) * s[:, :q.shape[1], :q.shape[2]]


def rms_norm(h, gamma, eps=1e-5):
    """y of rows [n][(lmax + 1)^2][C] already summed with their residual; gamma [lmax + 1][C]."""
    h, gamma = np.asarray(h, np.float64), np.asarray(gamma, np.float64)
    y = np.zeros(h.shape)
    with np.errstate(invalid="ignore"):
        for l in range(gamma.shape[0]):
            part = h[:, l * l:(l + 1) ** 2]
            y[:, l * l:(l + 1) ** 2] = part * gamma[l] / np.sqrt((part ** 2).mean((1, 2), keepdims=True) + eps)
    return y


def rms_norm_backward(h, dy, gamma, dh=None, eps=1e-5):
    """(dx, dgamma, sums of the magnitudes of the terms of each)."""
    h, dy, gamma = (np.asarray(a, np.float64) for a in (h, dy, gamma))
    dx, size = np.zeros(h.shape), np.zeros(h.shape)
    dgamma, terms = np.zeros(gamma.shape), np.zeros(gamma.shape)
    for l in range(gamma.shape[0]):
        at = slice(l * l, (l + 1) ** 2)
        v, d = h[:, at], dy[:, at] * gamma[l]
        rho = 1.0 / np.sqrt((v ** 2).mean((1, 2), keepdims=True) + eps)
        along = v * rho ** 2 * (d * v).mean((1, 2), keepdims=True)
        dx[:, at] = rho * (d - along)
        size[:, at] = rho * (np.abs(d) + np.abs(v) * rho ** 2 * np.abs(d * v).mean((1, 2), keepdims=True))
        dgamma[l], terms[l] = (dy[:, at] * v * rho).sum((0, 1)), np.abs(dy[:, at] * v * rho).sum((0, 1))
    if dh is not None:
        dx, size = dx + dh, size + np.abs(dh)
    return dx, dgamma, size, terms


def clip(tensors, most):
    """(norm, factor, scaled tensors); a norm that is not finite in fp32 scales nothing and gives the factor 0."""
    tensors = [np.asarray(t, np.float64) for t in tensors]
    norm = np.sqrt(sum((t ** 2).sum() for t in tensors))
    if not norm <= np.finfo(np.float32).max:
        return norm, 0.0, tensors
    factor = min(1.0, most / (norm + 1e-6))
    return norm, factor, [t * factor for t in tensors]
