"""Inputs, fp64 values and bounds of the group norm and its adjoint for their tests: how far each value of y and dx may be off, from that
value's own row, segment and group."""
import numpy as np

from oracle import block_oracle as K

U32 = 2.0 ** -24
HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
LEAST = {"float32": 2.0 ** -149, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -133}     # half a step of the smallest numbers, or one of theirs

# (rows, channels, groups, ends of segments or None, offset and scale of x unless they are 0.5 and 1.5)
CASES = [(1, 16, 4, None), (5, 12, 4, None), (333, 8, 1, None), (333, 33, 3, None), (333, 256, 8, None), (333, 1001, 7, None), (4095, 32, 4, None),
         (20001, 32, 4, None), (100001, 64, 8, None), (50000, 7, 1, None), (9000, 64, 8, [0, 9000, 9000]), (9000, 16, 4, [0, 0, 0, 9000]),
         (8192, 64, 8, [0, 2048, 4096, 6144, 8192]), (60000, 32, 4, [0, 7, 29999, 30000, 60000]), (900, 20, 4, [0, 4] + [7] * 60 + [900]),
         (901, 64, 8, list(range(0, 901, 3)) + [901]), (3000, 32, 4, None, 1000.0, 1.0)]


def inputs(case, seed=0):
    """x, dy, gamma, beta in fp64; dy has a mean and a part along x, so that both means of the adjoint are of order 1 however many rows."""
    (n, c), (offset, scale) = case[:2], case[4:] or (0.5, 1.5)
    groups = case[2]
    rng = np.random.default_rng([seed, n, c, groups])
    e = rng.standard_normal((n, c))
    dy = 0.7 + 0.5 * e + 0.3 * rng.standard_normal((n, c))
    return offset + scale * e, dy, (1 + 0.3 * rng.standard_normal(c)).astype(np.float32), (0.3 * rng.standard_normal(c)).astype(np.float32)


def adjoint(case, x, dy, gamma, beta, dtype, eps=1e-5):
    """(dx, bound, terms) from x and dy as they were given (fp64 values of the type); terms: rstd times (gamma dz, its mean, xhat times its mean with
    xhat), whose difference dx is.

    In steps of 2^-24, rounding by rounding: xhat = (x - mean) rstd takes one of the mean, and three of itself; z = gamma xhat + beta passes that on
    and adds two; dz = dy SiLU'(z) with |SiLU''| <= 1/2 adds 10 (1 + |z|) |dy| (exponential, reciprocal, products, 1 + z (1 - sig)); the means
    are off by the mean of what their terms are and 8 roundings of the terms (their sums); dx adds 6 of each of its terms and the
    rounding to its type."""
    n, c, groups, ptr = case[:4]
    _, mean, rstd = K.group_norm(x, groups, gamma, beta, ptr, eps)
    ptr = [0, n] if ptr is None else ptr
    size = c // groups
    dx, bound, terms = np.zeros((n, c)), np.zeros((n, c)), [np.zeros((n, c)) for _ in range(3)]
    for s, (b, e) in enumerate(zip(ptr[:-1], ptr[1:])):
        if e == b:
            continue
        def over(v):                       # mean over the segment's rows and the group's channels, back in every channel
            return np.repeat(v.reshape(e - b, groups, size).mean((0, 2)), size)
        mu, r = np.repeat(mean[s], size), np.repeat(rstd[s], size)
        h = (x[b:e] - mu) * r
        dh = U32 * (np.abs(mu) * r + 3 * np.abs(h))
        z = gamma * h + beta
        dz_off = np.abs(gamma) * dh + 2 * U32 * (np.abs(gamma * h) + np.abs(beta))
        sig = K.sigmoid(z)
        d = dy[b:e] * sig * (1 + z * (1 - sig))
        off = np.abs(dy[b:e]) * (0.5 * dz_off + 10 * U32 * (1 + np.abs(z)))
        gd, goff = gamma * d, np.abs(gamma) * off
        m1, m2 = over(gd), over(gd * h)
        m1_off = over(goff) + 8 * U32 * over(np.abs(gd))
        m2_off = over(goff * np.abs(h) + np.abs(gd) * dh) + 8 * U32 * over(np.abs(gd * h))
        parts = gd, np.broadcast_to(m1, gd.shape), h * m2
        for t, p in zip(terms, parts):
            t[b:e] = r * p
        dx[b:e] = r * (parts[0] - parts[1] - parts[2])
        bound[b:e] = r * (goff + m1_off + np.abs(h) * m2_off + np.abs(m2) * dh + 6 * U32 * sum(np.abs(p) for p in parts))
    return dx, bound * (1 + 2 * HALF_STEP[dtype]) + HALF_STEP[dtype] * np.abs(dx) + LEAST[dtype], terms


def forward(case, x, gamma, beta, dtype, eps=1e-5):
    """(y, bound): z as in adjoint(), |SiLU'| <= 1.1, and 6 + 2 |z| roundings of y (exponential, reciprocal, product)."""
    n, c, groups, ptr = case[:4]
    y, mean, rstd = K.group_norm(x, groups, gamma, beta, ptr, eps)
    ptr = [0, n] if ptr is None else ptr
    bound = np.zeros((n, c))
    for s, (b, e) in enumerate(zip(ptr[:-1], ptr[1:])):
        mu, r = np.repeat(mean[s], c // groups), np.repeat(rstd[s], c // groups)
        h = (x[b:e] - mu) * r
        z_off = U32 * (np.abs(gamma) * (np.abs(mu) * r + 3 * np.abs(h)) + 2 * (np.abs(gamma * h) + np.abs(beta)))
        bound[b:e] = 1.1 * z_off + U32 * (6 + 2 * np.abs(gamma * h + beta)) * np.abs(y[b:e])
    return y, bound * (1 + 2 * HALF_STEP[dtype]) + HALF_STEP[dtype] * np.abs(y) + LEAST[dtype]
