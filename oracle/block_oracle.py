"""fp64 oracle of the operators of a trained block: group norm with SiLU over ragged segments, rows times the matrix of their
group, orthogonalised updates.  Plain numpy from the formulas; no code shared with the library."""
import numpy as np

COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS_NORM_F = 1e-7


def sigmoid(z):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-z))


def group_norm(x, groups, gamma, beta, ptr=None, eps=1e-5):
    """(y, mean, rstd); rows of no segment stay NaN."""
    x = np.asarray(x, np.float64)
    n, c = x.shape
    ptr = [0, n] if ptr is None else ptr
    y = np.full((n, c), np.nan)
    mean, rstd = np.zeros((len(ptr) - 1, groups)), np.zeros((len(ptr) - 1, groups))
    for s in range(len(ptr) - 1):
        rows = x[ptr[s]:ptr[s + 1]]
        if not len(rows):
            continue
        v = rows.reshape(len(rows), groups, c // groups)
        mean[s] = v.mean((0, 2))
        rstd[s] = 1.0 / np.sqrt(v.var((0, 2)) + eps)
        z = ((v - mean[s][:, None]) * rstd[s][:, None]).reshape(rows.shape) * gamma + beta
        y[ptr[s]:ptr[s + 1]] = z * sigmoid(z)
    return y, mean, rstd


def group_norm_backward(x, dy, groups, gamma, beta, ptr=None, eps=1e-5):
    """(dx, dgamma, dbeta, sum |dy xhat|, sum |dy|); the last two say how far the sums in fewer bits may be off (|SiLU'| <= 1.1)."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    n, c = x.shape
    _, mean, rstd = group_norm(x, groups, gamma, beta, ptr, eps)
    ptr = [0, n] if ptr is None else ptr
    dx, terms_g, terms_b, hat = np.full((n, c), np.nan), np.zeros((n, c)), np.zeros((n, c)), np.zeros((n, c))
    for s in range(len(ptr) - 1):
        at = slice(ptr[s], ptr[s + 1])
        rows = len(x[at])
        if not rows:
            continue
        per = c // groups
        mu, r = np.repeat(mean[s], per), np.repeat(rstd[s], per)
        h = (x[at] - mu) * r
        z = h * gamma + beta
        sig = sigmoid(z)
        dz = dy[at] * sig * (1.0 + z * (1.0 - sig))
        terms_g[at], terms_b[at], hat[at] = dz * h, dz, h
        d = (dz * gamma).reshape(rows, groups, per)
        hg = h.reshape(rows, groups, per)
        v = d - d.mean((0, 2))[:, None] - hg * (d * hg).mean((0, 2))[:, None]
        dx[at] = v.reshape(rows, c) * r
    return dx, terms_g.sum(0), terms_b.sum(0), np.abs(dy * hat).sum(0), np.abs(dy).sum(0)


def group_rows(key, n_groups, lmax=-1):
    """(ptr, perm): rows by key, or the (lmax + 1)^2 rows of every atom by (key, degree), ascending inside a group."""
    key = np.clip(np.asarray(key, np.int64), 0, n_groups - 1)
    if lmax >= 0:
        degree = np.concatenate([np.full(2 * l + 1, l) for l in range(lmax + 1)])
        key = (key[:, None] * (lmax + 1) + degree).reshape(-1)
        n_groups *= lmax + 1
    perm = np.argsort(key, kind="stable")
    ptr = np.concatenate([[0], np.cumsum(np.bincount(key, minlength=n_groups))])
    return ptr.astype(np.int32), perm.astype(np.int32)


def grouped_linear(x, W, ptr, perm=None, bias=None):
    """(y, sum |terms|); rows of no group stay NaN."""
    x, W = np.asarray(x, np.float64), np.asarray(W, np.float64)
    n = x.shape[0]
    perm = np.arange(n) if perm is None else perm
    y, size = np.full((n, W.shape[1]), np.nan), np.full((n, W.shape[1]), np.nan)
    for g in range(W.shape[0]):
        rows = perm[ptr[g]:ptr[g + 1]]
        y[rows], size[rows] = x[rows] @ W[g].T, np.abs(x[rows]) @ np.abs(W[g]).T
        if bias is not None:
            y[rows] += bias[g]
            size[rows] += np.abs(bias[g])
    return y, size


def grouped_linear_backward(x, W, dy, ptr, perm=None):
    """(dx, dW, db) and the sums of their absolute terms."""
    x, W, dy = (np.asarray(a, np.float64) for a in (x, W, dy))
    n = x.shape[0]
    perm = np.arange(n) if perm is None else perm
    dx, dW, db = np.full(x.shape, np.nan), np.zeros(W.shape), np.zeros(W.shape[:2])
    sx, sW, sb = dx.copy(), dW.copy(), db.copy()
    for g in range(W.shape[0]):
        rows = perm[ptr[g]:ptr[g + 1]]
        d = dy[rows]
        dx[rows], dW[g], db[g] = d @ W[g], d.T @ x[rows], d.sum(0)
        a = np.abs(d)
        sx[rows], sW[g], sb[g] = a @ np.abs(W[g]), a.T @ np.abs(x[rows]), a.sum(0)
    return dx, dW, db, sx, sW, sb


def orthogonalise(g, steps=5):
    """The polynomial of the steps on the singular values: by products, from the side with fewer rows."""
    g = np.asarray(g, np.float64)
    a, b, c = COEFFICIENTS
    out = np.empty_like(g)
    for i in range(g.shape[0]):
        u = g[i] if g.shape[1] <= g.shape[2] else g[i].T
        x = u / (np.sqrt((u * u).sum()) + EPS_NORM_F)
        for _ in range(steps):
            p = x @ x.T
            x = a * x + b * (p @ x) + c * (p @ (p @ x))
        out[i] = x if g.shape[1] <= g.shape[2] else x.T
    return out


def muon_step(W, g, m, lr, beta=0.95, weight_decay=0.0, steps=5):
    W, g, m = (np.asarray(a, np.float64) for a in (W, g, m))
    m = beta * m + g
    o = orthogonalise(g + beta * m, steps)
    return (1.0 - lr * weight_decay) * W - lr * np.sqrt(max(1.0, W.shape[1] / W.shape[2])) * o, m
