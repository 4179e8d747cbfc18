"""Workspace sizes of a trained block's calls at the largest sizes they take (host arithmetic, no GPU needed)."""
import os

import pytest


@pytest.fixture(scope="module")
def m():
    from paper_2507_03840_amd import binding as B
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return B.Egnn(2, 32, 16, 10.0, 200.0)


@pytest.mark.parametrize("segments", [2 ** 30, 2 ** 31 - 513, 2 ** 31 - 1])
@pytest.mark.parametrize("rows", [1, 1000, 2 ** 31 - 1])
def test_group_norm_of_very_many_segments(m, rows, segments):
    """A pair of fp64 sums and a first value for every segment at least, and no more than two of them."""
    size = m.egnn_group_norm_workspace_bytes(rows, segments, 8, 2)
    assert 40 * segments <= size <= 80 * segments


def test_strides_of_what_is_not_there(m):
    """x is read for dW only and dx may be left out: their strides are looked at with them alone.  (Nothing to do, so nothing is launched.)"""
    def call(**change):
        a = dict(dtype=0, x=None, xs=0, W=None, dy=None, dys=16, n=0, k=32, out=16, ptr=4096, perm=None, g=3, dx=None, dxs=0, dW=None, db=None,
                 ws=4096, size=1 << 30, st=None)
        return m.lib.egnn_grouped_linear_backward(m.ctx, *dict(a, **change).values())
    assert call() == 0
    assert call(dys=15) == -1 and call(dx=4096) == -1 and call(dx=4096, dxs=32) == 0 and call(dW=4096, xs=31) == -1
