"""Operators of a trained block beside the message passing, as cases that can be timed and compared.

A block between two layers takes the scalar channels (or every row) of the node or edge embeddings through a group norm
with SiLU and through linear maps that depend on the species of the atom and on the degree of the row, and its weights
are trained with orthogonalised updates.  Kinds of case, and what each stands for in real use:
  norm          group norm with SiLU over the rows of a structure (or of each of several), channels last; inference
  norm_train    the same with its adjoint
  linear        rows times the matrix of their group; the structure is new, so the rows are put in groups in the pass
  linear_train  forward and adjoint (dx, dW, db); the rows' order by group is in hand, as it is between two steps
  orthogonal    an update orthogonalised by Newton-Schulz products
  muon          a step of the optimiser: momentum, orthogonalised update, new weights
Rows, channels and degrees are those of the library's configurations (64, 1,000, 3,000 and 12,000 + 8,000 atoms; 16, 32
and 64 channels; lmax 4; 625,262 and 2,350,179 edges) and generic odd ones.

With own = False everything is computed with elementary torch operations in 32 bits; exact() restates it in 64 bits.
"""
import math

import torch

own = False

COEFFICIENTS = (3.4445, -4.7750, 2.0315)   # of the quintic Newton-Schulz step, as published with the Muon optimiser
STEPS = 5
EPS_NORM = 1e-5
EPS_ORTHO = 1e-7
LR, BETA, DECAY = 0.02, 0.95, 0.01
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# ----------------------------------------------------------------------------------------------------------- cases
def _norm(name, rows, channels, groups, dtype="f32", segments=1, planes=1, train=False):
    """planes: the normalised rows are plane 0 of [rows][planes][channels]."""
    return dict(name=name, kind="norm_train" if train else "norm", rows=rows, channels=channels, groups=groups, dtype=dtype,
                segments=segments, planes=planes)


def _linear(name, rows, n_in, n_out, groups, dtype="f32", lmax=-1, empty=0, train=False):
    """lmax >= 0: rows is the number of atoms, whose (lmax + 1)^2 rows go by (species, degree): groups = species.
    empty: so many of the groups get no rows."""
    return dict(name=name, kind="linear_train" if train else "linear", rows=rows, n_in=n_in, n_out=n_out, groups=groups,
                dtype=dtype, lmax=lmax, empty=empty)


def _ortho(name, batch, rows, cols, dtype="f32", muon=True):
    return dict(name=name, kind="muon" if muon else "orthogonal", batch=batch, rows=rows, cols=cols, dtype=dtype)


def listed():
    return [
        # scalars of a molecule-sized cluster: launches and latency
        _norm("norm_64", 64, 16, 4),
        # scalar plane of a batch of ragged structures, read and written inside the node tensors of lmax 4
        _norm("norm_train_nodes_20000", 20000, 64, 8, segments=37, planes=25, train=True),
        # scalars of the edge embeddings of the 3,000-atom workload, a training step
        _norm("norm_train_edges_625262", 625262, 32, 4, train=True),
        # scalars of the edge embeddings of the slab in half the bytes, inference
        _norm("norm_edges_2350179_bf16", 2350179, 64, 8, dtype="bf16"),
        # a cluster's rows by species: launches and latency
        _linear("linear_64", 64, 16, 16, 2),
        # odd channel counts, groups without rows, half precision
        _linear("linear_5001_f16", 5001, 100, 77, 7, dtype="f16", empty=2),
        # node embeddings of the slab by species and degree, a training step
        _linear("linear_train_12000", 12000, 64, 64, 3, lmax=4, train=True),
        # wide hidden layers of experts, bf16, a training step; the largest product
        _linear("linear_train_experts_bf16", 20000, 512, 1024, 16, dtype="bf16", train=True),
        # the degrees' channel mixes of three layers, one step
        _ortho("muon_mixes_32", 15, 32, 32),
        # second matrices of the radial networks of three layers (42 paths x 64 channels by 64)
        _ortho("muon_radial_2688", 3, 2688, 64),
        # order-0 matrix of the SO(2) transform at lmax 4 and 64 channels (320 of 960)
        _ortho("muon_so2_320", 3, 320, 960),
        # a wide generic update in half the bytes
        _ortho("orthogonal_2048_bf16", 1, 2048, 1536, dtype="bf16", muon=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm_train", "linear", "linear", "linear_train", "linear_train", "orthogonal", "muon"))
    dtype = rng.choice(("f32", "f32", "bf16", "f16"))
    if kind.startswith("norm"):
        channels = rng.choice((8, 12, 16, 24, 32, 32, 64, 64, 96, 128, 200, 256))
        groups = rng.choice([g for g in (1, 2, 4, 6, 8, 16, 32, channels) if channels % g == 0])
        size = {"f32": 4, "f16": 2, "bf16": 2}[dtype]
        most = 1.5e8 / (channels * size) if kind == "norm" else 7.5e7 / (channels * size)
        planes = rng.choice((1, 1, 9, 25))
        rows = _log(rng, 1, most / planes)
        segments = 1 if rng.random() < 0.5 else _log(rng, 1, max(1, min(rows, 300)))
        c = _norm("", rows, channels, groups, dtype, segments, planes, kind == "norm_train")
    elif kind.startswith("linear"):
        lmax = rng.choice((-1, -1, -1, 2, 3, 4))
        if lmax < 0:
            n_in, n_out, groups = _log(rng, 8, 1024), _log(rng, 8, 1024), _log(rng, 1, 64)
            if rng.random() < 0.6:
                n_in, n_out = max(8, n_in // 8 * 8), max(8, n_out // 8 * 8)
        else:
            n_in = n_out = rng.choice((16, 32, 64, 128))
            groups = rng.choice((1, 2, 3, 4))
        per = 1 if lmax < 0 else (lmax + 1) ** 2
        rows = _log(rng, 1, max(2.0, min(2e4 * 512 * 1024 / (n_in * n_out), 6e6 / (n_in + n_out)) / per))
        c = _linear("", rows, n_in, n_out, groups, dtype, lmax, rng.choice((0, 0, groups // 3)), kind == "linear_train")
    else:
        rows, cols = _log(rng, 8, 2048), _log(rng, 8, 2048)
        n, m = min(rows, cols), max(rows, cols)
        batch = _log(rng, 1, max(1.0, min(32.0, 1.5e10 / (n * n * (3 * m + n)), 4e6 / (n * m))))
        c = _ortho("", batch, rows, cols, "f32" if kind == "muon" else dtype, kind == "muon")
    del c["name"]
    return c


# --------------------------------------------------------------------------------------------------------- inputs
def _gauss(seed, tag, shape, scale=1.0, dtype=torch.float32):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000 + tag)
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _ragged(n, parts):
    """parts + 1 offsets of n rows, lengths growing from part to part and some odd; the same for every seed."""
    w = torch.arange(1, parts + 1, dtype=torch.float64) + 0.37 * (torch.arange(parts) % 3)
    at = torch.floor(torch.cumsum(w, 0) / w.sum() * n).long()
    at[-1] = n
    return torch.cat([torch.zeros(1, dtype=torch.long), at])


def _keys(case, seed):
    """Group of every row; the groups' sizes depend on the case alone, the order on the seed."""
    full = case["groups"] - case["empty"]
    at = _ragged(case["rows"], full)
    key = torch.repeat_interleave(torch.arange(full) + case["empty"] // 2, at[1:] - at[:-1])
    gen = torch.Generator()
    gen.manual_seed(int(seed) * 1000 + 1)
    return key[torch.randperm(case["rows"], generator=gen)].to(torch.int32)


def _degrees(lmax):
    return torch.repeat_interleave(torch.arange(lmax + 1), 2 * torch.arange(lmax + 1) + 1).to(torch.int32)


def _row_keys(key, lmax):
    """(species, degree) of the rows of the atoms' embeddings."""
    if lmax < 0:
        return key
    return (key[:, None] * (lmax + 1) + _degrees(lmax).to(key.device)[None, :]).reshape(-1)


def _sizes(case):
    """Rows and groups of a product."""
    if case["lmax"] < 0:
        return case["rows"], case["groups"]
    return case["rows"] * (case["lmax"] + 1) ** 2, case["groups"] * (case["lmax"] + 1)


def _inputs(case, seed):
    s = dict(case=case)
    t = TYPES[case["dtype"]]
    if case["kind"].startswith("norm"):
        n, C = case["rows"], case["channels"]
        shape = (n, case["planes"], C)
        s["x"] = _gauss(seed, 2, shape, 1.5, t).add_(0.5)[:, 0]
        s["gamma"], s["beta"] = _gauss(seed, 3, (C,), 0.3).add_(1.0), _gauss(seed, 4, (C,), 0.3)
        s["at"] = _ragged(n, case["segments"]).tolist()
        s["ptr"] = torch.tensor(s["at"], dtype=torch.int32, device="cuda") if case["segments"] > 1 else None
        if case["kind"] == "norm_train":
            s["dy"] = _gauss(seed, 5, shape, 1.0, t)[:, 0]
    elif case["kind"].startswith("linear"):
        n, G = _sizes(case)
        K, N = case["n_in"], case["n_out"]
        s["x"] = _gauss(seed, 2, (n, K), 1.0, t)
        s["W"] = _gauss(seed, 3, (G, N, K), K ** -0.5, t)
        s["bias"] = _gauss(seed, 4, (G, N), 0.3)
        s["key"] = _keys(case, seed).cuda()
        if case["kind"] == "linear_train":
            s["dy"] = _gauss(seed, 5, (n, N), 1.0, t)
            row_key = _row_keys(s["key"], case["lmax"])
            s["perm"] = torch.sort(row_key, stable=True).indices.to(torch.int32)
            count = torch.bincount(row_key, minlength=G)
            s["ptr"] = torch.cat([count.new_zeros(1), torch.cumsum(count, 0)]).to(torch.int32)
            s["at"] = s["ptr"].tolist()
    else:
        shape = (case["batch"], case["rows"], case["cols"])
        # gradients of trained matrices: a few strong directions over many weak ones
        n, m, r = case["rows"], case["cols"], max(1, min(case["rows"], case["cols"]) // 8)
        g = _gauss(seed, 2, shape) + 2.0 * torch.matmul(_gauss(seed, 6, (case["batch"], n, r)), _gauss(seed, 7, (case["batch"], r, m)))
        g *= 1e-3 * math.sqrt(1.0 / (n + m))
        s["g"] = g.to(t)
        if case["kind"] == "muon":
            s["W"] = _gauss(seed, 3, shape, m ** -0.5)
            s["m"] = _gauss(seed, 4, shape, 1e-3 * math.sqrt(1.0 / (n + m)))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _keep(case, s)
    return s


def _keep(case, s):
    """Context, outputs and workspace that a program keeps from call to call."""
    from paper_2507_03840_amd import binding as B
    s["lib"] = m = B.Egnn(max(0, case.get("lmax", 0)), 32, 16, 10.0, 200.0)
    empty = lambda shape, t=torch.float32: torch.empty(shape, dtype=t, device="cuda")
    nbytes = 0
    if case["kind"].startswith("norm"):
        n, C, S = case["rows"], case["channels"], case["segments"]
        s["y"] = torch.empty_like(s["x"], memory_format=torch.contiguous_format)
        s["mean"], s["rstd"] = empty((S, case["groups"])), empty((S, case["groups"]))
        nbytes = m.egnn_group_norm_workspace_bytes(n, S, C, case["groups"])
        if case["kind"] == "norm_train":
            s["dx"] = torch.empty_like(s["y"])
            s["dgamma"], s["dbeta"] = empty((C,)), empty((C,))
    elif case["kind"].startswith("linear"):
        n, G = _sizes(case)
        s["y"] = empty((n, case["n_out"]), s["x"].dtype)
        if case["kind"] == "linear":
            s["ptr"], s["perm"] = empty((G + 1,), torch.int32), empty((n,), torch.int32)
            nbytes = m.egnn_group_rows_workspace_bytes(case["rows"], case["groups"])
        else:
            s["dx"], s["dW"], s["db"] = torch.empty_like(s["x"]), empty(s["W"].shape), empty(s["bias"].shape)
            nbytes = m.egnn_grouped_linear_workspace_bytes(n, G, case["n_in"], case["n_out"])
    else:
        s["out"] = torch.empty_like(s["g"])
        if case["kind"] == "muon":
            s["W_out"], s["m_out"] = torch.empty_like(s["W"]), torch.empty_like(s["m"])
        nbytes = m.egnn_orthogonalise_workspace_bytes(case["batch"], case["rows"], case["cols"])
    s["ws"] = torch.empty(max(256, nbytes), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------------ plain forms
def _norm_plain(s):
    case = s["case"]
    G, C = case["groups"], case["channels"]
    x = s["x"].float()
    y, mean, rstd = torch.empty_like(x), [], []
    xhat = torch.empty_like(x)
    at = s["at"]
    for b, e in zip(at[:-1], at[1:]):
        v = x[b:e].reshape(e - b, G, C // G)
        if e > b:
            mu = v.mean((0, 2))
            var = ((v - mu[:, None]) ** 2).mean((0, 2))
            r = (var + EPS_NORM) ** -0.5
        else:
            mu = r = torch.zeros(G, device=x.device)
        mean.append(mu)
        rstd.append(r)
        xhat[b:e] = ((v - mu[:, None]) * r[:, None]).reshape(e - b, C)
    z = xhat * s["gamma"] + s["beta"]
    sig = 1.0 / (1.0 + torch.exp(-z))
    out = dict(y=(z * sig).to(s["x"].dtype), mean=torch.stack(mean), rstd=torch.stack(rstd))
    if case["kind"] == "norm":
        return out
    dz = s["dy"].float() * (sig * (1.0 + z * (1.0 - sig)))
    out["dgamma"], out["dbeta"] = (dz * xhat).sum(0), dz.sum(0)
    dz = dz * s["gamma"]
    dx = torch.empty_like(x)
    for i, (b, e) in enumerate(zip(at[:-1], at[1:])):
        if e > b:
            d, h = dz[b:e].reshape(e - b, G, C // G), xhat[b:e].reshape(e - b, G, C // G)
            dv = (d - d.mean((0, 2))[:, None] - h * (d * h).mean((0, 2))[:, None]) * rstd[i][:, None]
            dx[b:e] = dv.reshape(e - b, C)
    out["dx"] = dx.to(s["x"].dtype)
    return out


def _linear_plain(s):
    case = s["case"]
    n, G = _sizes(case)
    if case["kind"] == "linear":
        row_key = _row_keys(s["key"], case["lmax"])
        perm = torch.sort(row_key, stable=True).indices
        at = [0] + torch.cumsum(torch.bincount(row_key, minlength=G), 0).tolist()
    else:
        perm, at = s["perm"].long(), s["at"]
    x, W = s["x"].float(), s["W"].float()
    y = torch.empty((n, case["n_out"]), device=x.device)
    for g in range(G):
        rows = perm[at[g]:at[g + 1]]
        y[rows] = x[rows] @ W[g].t() + s["bias"][g]
    out = dict(y=y.to(s["x"].dtype))
    if case["kind"] == "linear":
        return out
    dy = s["dy"].float()
    dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty_like(s["bias"])
    for g in range(G):
        rows = perm[at[g]:at[g + 1]]
        d = dy[rows]
        dx[rows] = d @ W[g]
        dW[g] = d.t() @ x[rows]
        db[g] = d.sum(0)
    return dict(out, dx=dx.to(s["x"].dtype), dW=dW, db=db)


def _orthogonalise(u):
    """[batch][rows][cols] -> the polynomial of the Newton-Schulz steps applied to its singular values."""
    a, b, c = COEFFICIENTS
    wide = u.shape[1] <= u.shape[2]
    x = (u if wide else u.transpose(1, 2)).contiguous()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS_ORTHO)
    for _ in range(STEPS):
        g = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * g + c * torch.matmul(g, g), x)
    return x if wide else x.transpose(1, 2).contiguous()


def _ortho_plain(s):
    case = s["case"]
    if case["kind"] == "orthogonal":
        return _orthogonalise(s["g"].float()).to(s["g"].dtype)
    m = BETA * s["m"] + s["g"]
    o = _orthogonalise(s["g"] + BETA * m)
    scale = LR * math.sqrt(max(1.0, case["rows"] / case["cols"]))
    return dict(W=(1.0 - LR * DECAY) * s["W"] - scale * o, m=m)


# ------------------------------------------------------------------------------------------------------- operators
def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        return _norm_plain(s) if kind.startswith("norm") else _linear_plain(s) if kind.startswith("linear") else _ortho_plain(s)
    m = s["lib"]
    if kind.startswith("norm"):
        m.egnn_group_norm(s["x"], case["groups"], s["gamma"], s["beta"], ptr=s["ptr"], eps=EPS_NORM, y=s["y"], mean=s["mean"],
                          rstd=s["rstd"], ws=s["ws"])
        out = dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
        if kind == "norm_train":
            m.egnn_group_norm_backward(s["x"], s["dy"], s["mean"], s["rstd"], case["groups"], s["gamma"], s["beta"], ptr=s["ptr"],
                                       dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"], ws=s["ws"])
            out.update(dgamma=s["dgamma"], dbeta=s["dbeta"], dx=s["dx"])
        return out
    if kind.startswith("linear"):
        if kind == "linear":
            m.egnn_group_rows(s["key"], case["groups"], lmax=case["lmax"], ptr=s["ptr"], perm=s["perm"], ws=s["ws"])
        m.egnn_grouped_linear(s["x"], s["W"], s["ptr"], perm=s["perm"], bias=s["bias"], y=s["y"])
        out = dict(y=s["y"])
        if kind == "linear_train":
            m.egnn_grouped_linear_backward(s["x"], s["W"], s["dy"], s["ptr"], perm=s["perm"], dx=s["dx"], dW=s["dW"], db=s["db"],
                                           ws=s["ws"])
            out.update(dx=s["dx"], dW=s["dW"], db=s["db"])
        return out
    if kind == "orthogonal":
        return m.egnn_orthogonalise(s["g"], steps=STEPS, y=s["out"], ws=s["ws"])
    m.egnn_muon_step(s["W"], s["g"], s["m"], LR, beta=BETA, weight_decay=DECAY, steps=STEPS, W_out=s["W_out"], momentum_out=s["m_out"],
                     ws=s["ws"])
    return dict(W=s["W_out"], m=s["m_out"])


def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    if case["kind"].startswith("norm"):
        n = case["rows"] * case["channels"]
        if case["kind"] == "norm":
            return dict(bytes=2 * n * size, flops=14 * n)
        return dict(bytes=4 * n * size, flops=45 * n)
    if case["kind"].startswith("linear"):
        n, G = _sizes(case)
        K, N = case["n_in"], case["n_out"]
        used = min(n, G - case["empty"] * G // case["groups"])      # groups with rows: whose matrices are read
        if case["kind"] == "linear":
            return dict(bytes=n * (K + N) * size + used * N * (K * size + 4), flops=2 * n * K * N)
        return dict(bytes=2 * n * (K + N) * size + 8 * n + N * (used * (K * size + 4) + G * 4 * (K + 1)), flops=6 * n * K * N)
    n, m = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # the two symmetric products have half their entries to compute
    flops = case["batch"] * STEPS * (n * n * m + n ** 3 + 2 * n * n * m)
    return dict(bytes=case["batch"] * n * m * (20 if case["kind"] == "muon" else 2 * size), flops=flops)


# ------------------------------------------------------------------------------------------------------ in 64 bits
def _norm64(case, seed):
    n, C, G = case["rows"], case["channels"], case["groups"]
    inputs = _inputs(case, seed)
    x, gamma, beta = (inputs[k].double().requires_grad_() for k in ("x", "gamma", "beta"))
    at = inputs["at"]
    part = torch.repeat_interleave(torch.arange(case["segments"]), torch.tensor(at[1:]) - torch.tensor(at[:-1])).cuda()
    with torch.set_grad_enabled(case["kind"] == "norm_train"):
        def mean_of(v):                       # over the rows of the structure and the channels of the group
            per_row = v.reshape(n, G, C // G).sum(2)
            total = torch.zeros((case["segments"], G), dtype=torch.float64, device="cuda").index_add(0, part, per_row)
            size = torch.bincount(part, minlength=case["segments"]).double()[:, None] * (C // G)
            return total / size.clamp(min=1)
        mean = mean_of(x)
        centred = x - mean[part].repeat_interleave(C // G, 1)
        empty = (torch.bincount(part, minlength=case["segments"]) == 0)[:, None]
        rstd = torch.where(empty, torch.zeros_like(mean), 1.0 / torch.sqrt(mean_of(centred * centred) + EPS_NORM))
        z = centred * rstd[part].repeat_interleave(C // G, 1) * gamma + beta
        y = z * torch.sigmoid(z)
    out = dict(y=y.detach(), mean=mean.detach(), rstd=rstd.detach())
    if case["kind"] == "norm_train":
        dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), inputs["dy"].double())
        out.update(dgamma=dgamma, dbeta=dbeta, dx=dx)
    return out


def _linear64(case, seed):
    n, G = _sizes(case)
    inputs = _inputs(case, seed)
    x, W, bias = inputs["x"].double(), inputs["W"].double(), inputs["bias"].double()
    key = _row_keys(inputs["key"], case["lmax"])
    y = torch.zeros((n, case["n_out"]), dtype=torch.float64, device="cuda")
    train = case["kind"] == "linear_train"
    if train:
        dy = inputs["dy"].double()
        dx, dW, db = torch.zeros_like(x), torch.zeros_like(W), torch.zeros_like(bias)
    for g in range(G):
        mine = torch.nonzero(key == g)[:, 0]
        y[mine] = torch.addmm(bias[g], x[mine], W[g].t())
        if train:
            dx[mine] = torch.mm(dy[mine], W[g])
            dW[g] = torch.mm(dy[mine].t(), x[mine])
            db[g] = dy[mine].sum(0)
    return dict(y=y, dx=dx, dW=dW, db=db) if train else dict(y=y)


def _ortho64(case, seed):
    n, m = case["rows"], case["cols"]
    inputs = _inputs(case, seed)
    u = inputs["g"].double()
    if case["kind"] == "muon":
        momentum = inputs["m"].double() * BETA + u
        u = u + BETA * momentum
    out = torch.empty_like(u)
    for i in range(case["batch"]):
        x = u[i] / (torch.linalg.matrix_norm(u[i]) + EPS_ORTHO)
        for _ in range(STEPS):                # p(x) = a x + b (x x^T) x + c (x x^T)^2 x, from the side with fewer rows
            if n <= m:
                g = x @ x.t()
                x = COEFFICIENTS[0] * x + COEFFICIENTS[1] * (g @ x) + COEFFICIENTS[2] * (g @ (g @ x))
            else:
                g = x.t() @ x
                x = COEFFICIENTS[0] * x + COEFFICIENTS[1] * (x @ g) + COEFFICIENTS[2] * ((x @ g) @ g)
        out[i] = x
    if case["kind"] == "orthogonal":
        return out
    W = inputs["W"].double()
    return dict(W=W * (1.0 - LR * DECAY) - out * (LR * math.sqrt(max(1.0, n / m))), m=momentum)


def exact(case, seed):
    kind = case["kind"]
    return _norm64(case, seed) if kind.startswith("norm") else _linear64(case, seed) if kind.startswith("linear") else _ortho64(case, seed)
