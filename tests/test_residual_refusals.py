"""What the calls of a residual block refuse, and their workspace sizes: host checks, nothing is launched (no GPU needed)."""
import ctypes
import os

import pytest

# (made-up addresses stay off machines with a GPU)
pytestmark = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="host checks, run where there is no GPU")
F32, F16, BF16, EINVAL, EWS = 0, 1, 2, -1, -3
P, WS = 4096, 1 << 30     # never read: every call below is refused first


@pytest.fixture(scope="module")
def m():
    from paper_2507_03840_amd import binding as B
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return B.Egnn(2, 32, 16, 10.0, 200.0)


def refused(m, call, good, code, **change):
    assert getattr(m.lib, call)(m.ctx, *dict(good, **change).values()) == code, (call, change)
    assert m.lib.egnn_last_error(m.ctx)


NORM = dict(dtype=F32, x=P, xs=288, r=P, rs=288, n=10, lmax=2, c=32, gamma=P, eps=1e-5, h=2 * P, hs=288, y=3 * P, ys=288, q=P, qs=32, scale=P, st=None)
ADJOINT = dict(dtype=BF16, h=P, hs=288, dy=P, dys=288, dh=P, dhs=288, n=10, lmax=2, c=32, gamma=P, eps=1e-5, dx=P, dxs=288, dg=P, ws=P, size=WS, st=None)


@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(dtype=-1), dict(x=None), dict(xs=287), dict(rs=287), dict(n=-1), dict(n=2 ** 31), dict(lmax=-1), dict(lmax=16), dict(c=0),
    dict(c=65537), dict(gamma=None), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(hs=287), dict(ys=287),
    dict(h=P, r=None), dict(h=P, y=P), dict(y=None, q=None, scale=None), dict(q=None), dict(scale=None), dict(qs=31), dict(qs=40), dict(q=P + 8),
    dict(h=P, hs=300), dict(y=P, ys=300, h=None), dict(r=4 * P, y=4 * P, ys=289)])
def test_rms_norm(m, change):
    refused(m, "egnn_rms_norm", NORM, EINVAL, **change)


def test_rms_norm_backward(m):
    for change in (dict(dtype=3), dict(h=None), dict(dy=None), dict(dx=None), dict(dg=None), dict(gamma=None), dict(hs=287), dict(dys=287), dict(dhs=0),
                   dict(dxs=287), dict(n=-1), dict(n=2 ** 31), dict(lmax=-1), dict(lmax=16), dict(c=0), dict(c=65537), dict(eps=0.0), dict(dxs=300),
                   dict(dx=2 * P, dy=2 * P, dys=300), dict(dx=2 * P, dh=2 * P, dhs=290)):
        refused(m, "egnn_rms_norm_backward", ADJOINT, EINVAL, **change)
    for change in (dict(ws=None), dict(ws=P + 16), dict(size=100)):
        refused(m, "egnn_rms_norm_backward", ADJOINT, EWS, **change)


def test_quantise(m):
    good = dict(dtype=F32, x=P, xs=40, n=10, cols=40, q=P, qs=48, scale=P, st=None)
    for change in (dict(dtype=3), dict(x=None), dict(xs=39), dict(n=-1), dict(n=2 ** 31), dict(cols=0), dict(cols=65537), dict(q=None), dict(qs=32),
                   dict(qs=40), dict(q=P + 4), dict(scale=None)):
        refused(m, "egnn_quantise_rows", good, EINVAL, **change)
    good = dict(dtype=F16, W=P, batch=3, rows=40, cols=24, q=P, qs=32, scale=P, qt=P, ts=48, scale_t=P, st=None)
    for change in (dict(dtype=9), dict(W=None), dict(batch=-1), dict(batch=65536), dict(rows=0), dict(rows=65537), dict(cols=0), dict(cols=65537),
                   dict(q=None), dict(qs=16), dict(qs=24), dict(q=P + 1), dict(scale=None), dict(qt=None), dict(scale_t=None), dict(ts=32),
                   dict(ts=40), dict(qt=P + 8), dict(batch=65535, rows=65536, cols=65536, qs=65536, ts=65536)):
        refused(m, "egnn_quantise_matrices", good, EINVAL, **change)


def test_scaled_linear(m):
    good = dict(q=P, qs=48, scale=P, n=10, k=40, out=24, w=P, ws=48, wscale=P, b=P, ptr=P, perm=P, g=3, dtype=BF16, y=P, ys=24, st=None)
    for change in (dict(q=None), dict(qs=32), dict(qs=40), dict(q=P + 8), dict(scale=None), dict(n=-1), dict(n=2 ** 31), dict(k=0), dict(k=65537), dict(out=0),
                   dict(out=65537), dict(w=None), dict(ws=32), dict(ws=44), dict(w=P + 4), dict(wscale=None), dict(ptr=None), dict(ptr=None, g=1),
                   dict(g=0), dict(g=65536), dict(dtype=3), dict(y=None), dict(ys=23)):
        refused(m, "egnn_scaled_linear", good, EINVAL, **change)


def tensors(*rows):
    from paper_2507_03840_amd import binding as B
    return (B.TensorDesc * len(rows))(*(B.TensorDesc(*r, 0) for r in rows))


def test_clip_gradients(m):
    def call(t, count=None, most=1.0, norm=P, ws=P, size=WS):
        return m.lib.egnn_clip_gradients(m.ctx, ctypes.addressof(t) if t is not None else None, len(t) if count is None else count, most, norm, ws, size, None)
    good = (1 << 20, 2 << 20, 100, F32)
    for t in ([(None, P, 5, F32)], [(P, None, 5, F32)], [(P, P, -1, F32)], [(P, P, 2 ** 40 + 1, F32)], [(P, P, 5, 3)], [(P + 2, P + 2, 5, F32)], [(P + 1, P, 5, BF16)]):
        assert call(tensors(*t)) == EINVAL and call(tensors(good, *t)) == EINVAL, t
    assert call(None, 1) == EINVAL and call(tensors(good), -1) == EINVAL
    for most in (0.0, -1.0, float("nan")):
        assert call(tensors(good), most=most) == EINVAL
    assert call(tensors(good), norm=None) == EINVAL
    for change in (dict(ws=None), dict(ws=P + 8), dict(size=7)):
        assert call(tensors(good), **change) == EWS


@pytest.mark.parametrize("rows", [
    [(P, P, 100, F32), (P, P, 100, F32)],                          # the same tensor twice
    [(P, 2 * P, 100, F32), (3 * P, 2 * P, 100, F32)],              # two results at one place
    [(P, 2 * P, 100, F32), (2 * P, 3 * P, 100, F32)],              # a result over another tensor
    [(P, P + 4, 100, F32)],                                        # a result beside its own source
    [(P, P, 100, F32), (P + 396, 9 * P, 1, F32)],                  # one value shared
    [(P, 2 * P, 100, BF16), (P, 3 * P, 100, BF16), (P + 100, P + 100, 10, BF16)]])
def test_clip_gradients_refuses_overlaps(m, rows):
    t = tensors(*rows)
    assert m.lib.egnn_clip_gradients(m.ctx, ctypes.addressof(t), len(t), 1.0, P, P, WS, None) == EINVAL
    assert b"overlaps" in m.lib.egnn_last_error(m.ctx)


def test_workspaces(m):
    from paper_2507_03840_amd import binding as B
    for args in ((-1, 0, 8), (2 ** 31, 0, 8), (5, -1, 8), (5, 16, 8), (5, 0, 0), (5, 0, 65537)):
        with pytest.raises(B.EgnnError) as e:
            m.egnn_rms_norm_workspace_bytes(*args)
        assert e.value.code == EINVAL
    assert m.egnn_rms_norm_workspace_bytes(0, 4, 64) >= 0
    assert m.egnn_rms_norm_workspace_bytes(2 ** 31 - 1, 15, 65536) < 2 ** 40
    n = ctypes.c_size_t()
    t = tensors((P, P, 2 ** 40, BF16), (P, P, 0, F32), (None, None, 0, F16))
    assert m.lib.egnn_clip_gradients_workspace_bytes(m.ctx, ctypes.addressof(t), 3, ctypes.addressof(n)) == 0 and 0 < n.value < 1 << 20
    assert m.lib.egnn_clip_gradients_workspace_bytes(m.ctx, None, 0, ctypes.addressof(n)) == 0 and n.value == 0
    assert m.lib.egnn_clip_gradients_workspace_bytes(m.ctx, None, 1, ctypes.addressof(n)) == EINVAL
    assert m.lib.egnn_clip_gradients_workspace_bytes(m.ctx, ctypes.addressof(t), 3, None) == EINVAL


def test_nothing_to_do_is_no_error(m):
    """No rows and no matrices: nothing is launched, whatever the addresses."""
    assert m.lib.egnn_rms_norm(m.ctx, *dict(NORM, n=0, x=None, r=None, h=None, y=None, q=None, scale=None).values()) == 0
    assert m.lib.egnn_quantise_rows(m.ctx, F32, None, 8, 0, 8, None, 16, None, None) == 0
    assert m.lib.egnn_quantise_matrices(m.ctx, F32, None, 0, 8, 8, None, 16, None, None, 0, None, None) == 0
    assert m.lib.egnn_scaled_linear(m.ctx, None, 16, None, 0, 8, 8, P, 16, P, None, None, None, 1, F32, None, 8, None) == 0


def test_binding_refuses_tensors_that_do_not_fit(m):
    """Before anything reaches the library: host tensors, wrong types and shapes."""
    import torch
    from paper_2507_03840_amd import binding as B
    x, gamma, three = torch.zeros(10, 9, 32), torch.ones(3, 32), torch.zeros(10, 1, 32)
    q, s = B.empty_codes((10, 32), "cpu")
    w, ws = B.empty_matrix_codes((1, 8, 32), "cpu")
    host = torch.zeros(256, dtype=torch.uint8)
    for call in (lambda: m.egnn_rms_norm(x, gamma), lambda: m.egnn_rms_norm(x.double(), gamma), lambda: m.egnn_rms_norm(x[:, :8], gamma),
                 lambda: m.egnn_rms_norm(three, gamma), lambda: m.egnn_rms_norm(x, gamma, h=x), lambda: m.egnn_rms_norm_backward(x, x, gamma, dx=x, dgamma=gamma, ws=host),
                 lambda: m.egnn_rms_norm_backward(x[0], x[0], gamma), lambda: m.egnn_quantise_rows(x[:, 0]), lambda: m.egnn_quantise_rows(x[:, 0], q=q),
                 lambda: m.egnn_quantise_matrices(torch.zeros(1, 3, 4)), lambda: m.egnn_quantise_matrices(torch.zeros(1, 3, 4), qt=q),
                 lambda: m.egnn_scaled_linear(q, s, w, ws, y=x[:, 0]), lambda: m.egnn_clip_gradients([x], 1.0, norm=x, ws=host), lambda: m.egnn_clip_gradients([x.int()], 1.0),
                 lambda: B.TensorList([x], [])):
        with pytest.raises(ValueError):
            call()


def test_places_of_codes():
    """Rows from multiples of 16 bytes on, whatever their length; strides that are no such rows are refused."""
    from paper_2507_03840_amd import binding as B
    for n in (1, 15, 16, 17, 128, 129):
        q, s = B.empty_codes((3, 4, n), "cpu")
        assert q.shape == (3, 4, n) and q.stride() == (4 * (-(-n // 16) * 16), -(-n // 16) * 16, 1) and s.shape == (3, 4, -(-n // 128))
        w, ws = B.empty_matrix_codes((2, 130, n), "cpu")
        assert w.stride() == (130 * (-(-n // 16) * 16), -(-n // 16) * 16, 1) and ws.shape == (2, 2, -(-n // 128))


def test_tensors_of_another_device_are_refused(monkeypatch):
    from types import SimpleNamespace
    from paper_2507_03840_amd import binding as B
    monkeypatch.setattr(B, "_device", lambda: 0)
    on = lambda k: SimpleNamespace(get_device=lambda: k, device=f"cuda:{k}")
    B._here(on(0), None, False, on(0), on(-1))
    with pytest.raises(ValueError, match="cuda:1"):
        B._here(on(0), None, on(1))


def test_addresses_of_tensors_without_values_are_not_looked_at(m):
    n = ctypes.c_size_t()
    for dtype in (F32, BF16):
        t = tensors((P, P, 10, F32), (P + 1, P + 3, 0, dtype), (None, P + 1, 0, dtype))
        assert m.lib.egnn_clip_gradients_workspace_bytes(m.ctx, ctypes.addressof(t), 3, ctypes.addressof(n)) == 0 and n.value > 0


def test_a_list_of_tensors_from_a_generator():
    """What can be gone through once is gone through once: results go to the tensors themselves."""
    import torch
    from paper_2507_03840_amd import binding as B

    class Device:                                  # what the list asks of a device tensor
        is_cuda, dtype = True, torch.float32

        def __init__(self, at, n):
            self.at, self.shape, self.n = at, torch.Size((n,)), n

        is_contiguous = lambda self: True
        data_ptr = lambda self: self.at
        numel = lambda self: self.n
        get_device = lambda self: 0

    tensors = [Device(P, 5), Device(2 * P, 7), Device(3 * P, 0)]
    got = B.TensorList(t for t in tensors)
    assert got.tensors == tensors and got.out == tensors and got.device == 0
    assert [(d.data, d.out, d.n, d.dtype) for d in got.desc] == [(P, P, 5, F32), (2 * P, 2 * P, 7, F32), (3 * P, 3 * P, 0, F32)]
    elsewhere = [Device(k * P, t.n) for k, t in enumerate(tensors, 5)]
    got = B.TensorList((t for t in tensors), (t for t in elsewhere))
    assert [(d.data, d.out) for d in got.desc] == [(P, 5 * P), (2 * P, 6 * P), (3 * P, 7 * P)]
    for out in ((t for t in elsewhere[:2]), (t for t in ())):
        with pytest.raises(ValueError, match="places for results"):
            B.TensorList((t for t in tensors), out)
