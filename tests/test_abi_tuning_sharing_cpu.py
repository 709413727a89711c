"""Outputs that share memory are refused in calls without rows too, where they are the only memory that is written."""
from test_abi_tuning_cpu import AT, L, norm_backward, preference, shared  # noqa: F401


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


def test_losses_of_no_rows(L):  # noqa: F811
    none = dict(rows=0, offsets=AT, logp=AT * 2)
    assert shared(preference(L, **none, loss=AT * 2 + 12)) and not shared(preference(L, **none, loss=AT * 2 + 16))
    assert shared(preference(L, **none, ref=AT * 2)) and shared(preference(L, **none, weight=AT * 2 + 12))
    assert shared(preference(L, **none, loss=AT + 36)) and not shared(preference(L, **none, loss=AT + 40))
    # what has no memory shares none
    assert not shared(preference(L, **none, z=AT * 2, dz=AT * 2, ld_d=72, target=AT * 2, ws=AT * 2, ws_bytes=0))
    assert shared(preference(L, **none, ws=AT * 2 - 256, ws_bytes=260))
