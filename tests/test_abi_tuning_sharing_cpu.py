"""Outputs that share memory are refused in calls without rows too, where they are the only memory that is written."""
from test_abi_tuning_cpu import AT, L, norm_backward, shared  # noqa: F401


def test_norm_gradients_of_no_rows(L):  # noqa: F811
    none = dict(rows=0, h=AT, dy=AT)
    for acc in (0, 1):
        assert shared(norm_backward(L, **none, acc=acc, dgain=AT * 3, dbias=AT * 3)) and shared(norm_backward(L, **none, acc=acc, dgain=AT * 3, dbias=AT * 3 + 236))
        assert shared(norm_backward(L, **none, acc=acc, dgain=AT * 3, gain=AT * 3 + 232))
        assert not shared(norm_backward(L, **none, acc=acc, dgain=AT * 3, dbias=AT * 3 + 240))
    # what has no memory shares none: matrices and statistics of no rows, a workspace of no bytes
    assert not shared(norm_backward(L, rows=0, h=AT, dy=AT + 16, dx=AT + 32, ld_h=64, ld_dx=72, mean=AT, rstd=AT, dgain=AT, mask=AT))
    assert not shared(norm_backward(L, **none, dgain=AT * 3, ws=AT * 3 + 16, ws_bytes=0))
    assert shared(norm_backward(L, **none, dgain=AT * 3, ws=AT * 3 + 16, ws_bytes=256))
