"""What the calls of a trained block refuse, and their workspace sizes: host checks, nothing is launched (no GPU needed)."""
import ctypes
import re
import os

import pytest

# (made-up addresses stay off machines with a GPU)
pytestmark = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="host checks, run where there is no GPU")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, F16, BF16, EINVAL, EWS = 0, 1, 2, -1, -3
P, WS = 4096, 1 << 20     # never read: every call below is refused first


@pytest.fixture(scope="module")
def m():
    from paper_2507_03840_amd import binding as B
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return B.Egnn(2, 32, 16, 10.0, 200.0)


def test_argument_types_follow_the_header(m):
    from paper_2507_03840_amd import binding as B
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "egnn.h")).read(), flags=re.S)
    for name, letters in B._SIGNATURES.items():
        args = re.search(r"int " + name + r"\((.*?)\);", header, re.S).group(1).split(",")
        kind = lambda a: "p" if "*" in a else {"int32_t": "i", "int64_t": "l", "float": "f", "size_t": "z"}[a.split()[-2]]
        assert "".join(kind(a) for a in args) == letters, name


def refused(m, call, good, code, **change):
    args = dict(good, **change)
    assert getattr(m.lib, call)(m.ctx, *args.values()) == code, (call, change)
    assert m.lib.egnn_last_error(m.ctx)


def test_group_norm(m):
    good = dict(dtype=F32, x=P, xs=32, n=100, c=32, g=4, ptr=P, s=2, gamma=P, beta=P, eps=1e-5, y=P, ys=32, mean=P, rstd=P, ws=P, size=WS, st=None)
    for change in (dict(dtype=3), dict(dtype=-1), dict(n=-1), dict(n=2 ** 31), dict(c=0), dict(c=1025), dict(g=0), dict(g=5), dict(s=0),
                   dict(ptr=None), dict(gamma=None), dict(beta=None), dict(mean=None), dict(rstd=None), dict(x=None), dict(y=None),
                   dict(xs=31), dict(ys=31), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan"))):
        refused(m, "egnn_group_norm", good, EINVAL, **change)
    for change in (dict(ws=None), dict(ws=P + 16), dict(size=0)):
        refused(m, "egnn_group_norm", good, EWS, **change)
    good = dict(dtype=BF16, x=P, xs=32, dy=P, dys=32, mean=P, rstd=P, n=100, c=32, g=4, ptr=P, s=2, gamma=P, beta=P, dx=P, dxs=32, dg=P, db=P,
                ws=P, size=WS, st=None)
    for change in (dict(dtype=7), dict(n=-1), dict(c=33), dict(g=0), dict(s=0), dict(ptr=None), dict(x=None), dict(dy=None), dict(dx=None),
                   dict(mean=None), dict(rstd=None), dict(gamma=None), dict(beta=None), dict(dg=None), dict(db=None), dict(xs=31), dict(dys=0),
                   dict(dxs=-32)):
        refused(m, "egnn_group_norm_backward", good, EINVAL, **change)
    for change in (dict(ws=None), dict(ws=P + 16), dict(size=255)):
        refused(m, "egnn_group_norm_backward", good, EWS, **change)


def test_group_rows(m):
    good = dict(key=P, n=100, g=4, lmax=2, ptr=P, perm=P, ws=P, size=WS, st=None)
    for change in (dict(key=None), dict(n=-1), dict(n=2 ** 31 // 9 + 1), dict(g=0), dict(g=1025), dict(lmax=-2), dict(lmax=16), dict(ptr=None),
                   dict(perm=None)):
        refused(m, "egnn_group_rows", good, EINVAL, **change)
    for change in (dict(ws=None), dict(ws=P + 8), dict(size=15)):
        refused(m, "egnn_group_rows", good, EWS, **change)


def test_grouped_linear(m):
    good = dict(dtype=F16, x=P, xs=32, n=100, k=32, out=16, W=P, b=P, ptr=P, perm=P, g=3, y=P, ys=16, st=None)
    for change in (dict(dtype=9), dict(x=None), dict(xs=31), dict(n=-1), dict(n=2 ** 31), dict(k=0), dict(k=65537), dict(out=0), dict(out=65537),
                   dict(W=None), dict(ptr=None), dict(g=0), dict(g=65536), dict(y=None), dict(ys=15)):
        refused(m, "egnn_grouped_linear", good, EINVAL, **change)
    good = dict(dtype=F32, x=P, xs=32, W=P, dy=P, dys=16, n=100, k=32, out=16, ptr=P, perm=P, g=3, dx=P, dxs=32, dW=P, db=P, ws=P, size=1 << 30,
                st=None)
    for change in (dict(dtype=9), dict(x=None), dict(xs=31), dict(W=None), dict(dy=None), dict(dys=15), dict(n=-1), dict(k=0), dict(out=0),
                   dict(ptr=None), dict(g=0), dict(dxs=31)):
        refused(m, "egnn_grouped_linear_backward", good, EINVAL, **change)
    for change in (dict(ws=None), dict(ws=P + 8), dict(size=0)):
        refused(m, "egnn_grouped_linear_backward", good, EWS, **change)


def test_orthogonalise_and_muon(m):
    good = dict(dtype=F32, g=P, batch=2, rows=8, cols=9, steps=5, y=P, ws=P, size=1 << 30, st=None)
    for change in (dict(dtype=4), dict(g=None), dict(batch=-1), dict(batch=65536), dict(rows=0), dict(rows=65537), dict(cols=0), dict(cols=65537),
                   dict(steps=0), dict(steps=33), dict(y=None)):
        refused(m, "egnn_orthogonalise", good, EINVAL, **change)
    for change in (dict(ws=None), dict(ws=P + 8), dict(size=0)):
        refused(m, "egnn_orthogonalise", good, EWS, **change)
    good = dict(W=P, g=P, mom=P, batch=2, rows=8, cols=9, lr=0.1, beta=0.9, wd=0.0, steps=5, Wo=P, mo=P, ws=P, size=1 << 30, st=None)
    for change in (dict(W=None), dict(g=None), dict(mom=None), dict(Wo=None), dict(mo=None), dict(steps=0), dict(batch=-2), dict(rows=0), dict(cols=0)):
        refused(m, "egnn_muon_step", good, EINVAL, **change)
    for change in (dict(ws=None), dict(ws=P + 8), dict(size=0)):
        refused(m, "egnn_muon_step", good, EWS, **change)


def test_workspace_calls(m):
    from paper_2507_03840_amd import binding as B
    for call, args in ((m.egnn_group_norm_workspace_bytes, (10, 1, 32, 5)), (m.egnn_group_norm_workspace_bytes, (-1, 1, 32, 4)),
                       (m.egnn_group_rows_workspace_bytes, (5, 0)), (m.egnn_grouped_linear_workspace_bytes, (5, 0, 3, 3)),
                       (m.egnn_orthogonalise_workspace_bytes, (1, 0, 3))):
        with pytest.raises(B.EgnnError) as e:
            call(*args)
        assert e.value.code == EINVAL
    assert m.egnn_group_norm_workspace_bytes(0, 3, 32, 4) >= 0
    assert m.egnn_orthogonalise_workspace_bytes(0, 3, 32) >= 0
    n = ctypes.c_size_t()
    assert m.lib.egnn_group_rows_workspace_bytes(m.ctx, 5, 2, None) == EINVAL
    assert m.lib.egnn_group_rows_workspace_bytes(None, 5, 2, ctypes.addressof(n)) == EINVAL


def test_binding_refuses_tensors_that_do_not_fit(m):
    """Before anything reaches the library: host tensors, wrong types, shapes, strides."""
    import torch
    x, one = torch.zeros(10, 32), torch.ones(32)
    for call in (lambda: m.egnn_group_norm(x, 4, one, one, ws=torch.zeros(9, dtype=torch.uint8)),
                 lambda: m.egnn_group_norm(x.double(), 4, one, one),
                 lambda: m.egnn_grouped_linear(x, torch.zeros(2, 8, 32), torch.zeros(3, dtype=torch.int32)),
                 lambda: m.egnn_orthogonalise(torch.zeros(2, 3, 4, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()
