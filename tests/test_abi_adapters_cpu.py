"""Refusals and size queries of the adapter, dropout and token-loss entry points that need no GPU: every call here
returns from host-side validation."""
import pytest

import paper_2405_13954_amd as P

NULL = None


@pytest.fixture(scope="module")
def L():
    return P.lib()


def forward(L, **kw):
    a = dict(x=NULL, ld_x=64, dtype=1, rows=4, n_in=64, n_out=32, rank=8, n=2, plan=NULL, plan_bytes=0, A=NULL, B=NULL,
             scale=NULL, base=NULL, ld_base=32, y=NULL, ld_y=32, u=NULL, p=0.0, seed=1, offset=2, ws=NULL, ws_bytes=0, st=NULL)
    return L.logra_adapter_forward(*{**a, **kw}.values())


def backward(L, **kw):
    a = dict(x=NULL, ld_x=64, dy=NULL, ld_dy=32, dtype=1, rows=4, n_in=64, n_out=32, rank=8, n=2, plan=NULL, plan_bytes=0,
             A=NULL, B=NULL, scale=NULL, u=NULL, base=NULL, ld_base=64, dx=NULL, ld_dx=64, dA=NULL, dB=NULL, acc=0, p=0.0,
             seed=1, offset=2, ws=NULL, ws_bytes=0, st=NULL)
    return L.logra_adapter_backward(*{**a, **kw}.values())


BAD = [(dict(dtype=2), P.ERR_INVALID_ARG), (dict(rows=-1), P.ERR_INVALID_ARG), (dict(n_in=0), P.ERR_INVALID_ARG),
       (dict(n_in=60), P.ERR_INVALID_ARG), (dict(n_out=36), P.ERR_INVALID_ARG), (dict(dtype=0, n_out=30), P.ERR_INVALID_ARG),
       (dict(rank=0), P.ERR_INVALID_ARG), (dict(rank=129), P.ERR_UNSUPPORTED), (dict(n=0), P.ERR_INVALID_ARG),
       (dict(n=1024), P.ERR_UNSUPPORTED), (dict(rows=(1 << 24) + 1), P.ERR_UNSUPPORTED), (dict(ld_x=56), P.ERR_INVALID_ARG),
       (dict(ld_x=65), P.ERR_INVALID_ARG), (dict(p=1.0), P.ERR_INVALID_ARG), (dict(p=float("nan")), P.ERR_INVALID_ARG),
       (dict(p=-0.5), P.ERR_INVALID_ARG), (dict(p=1.0 - 1e-9), P.ERR_INVALID_ARG), (dict(n_in=1 << 21), P.ERR_UNSUPPORTED),
       (dict(ld_x=1 << 62), P.ERR_INVALID_ARG), (dict(), P.ERR_INVALID_ARG)]   # the last: null pointers


@pytest.mark.parametrize("change,status", BAD)
def test_adapter_refusals(L, change, status):
    assert forward(L, **change) == status
    assert backward(L, **change) == status
    assert P.logra_last_error()


def test_adapter_strides_and_no_rows(L):
    assert forward(L, ld_y=24) == P.ERR_INVALID_ARG and forward(L, ld_y=33) == P.ERR_INVALID_ARG
    assert backward(L, ld_dy=24) == P.ERR_INVALID_ARG
    assert backward(L, base=16) == P.ERR_INVALID_ARG and "without dx" in P.logra_last_error()
    assert forward(L, rows=0) == P.OK
    assert backward(L, rows=0) == P.ERR_INVALID_ARG and "dA" in P.logra_last_error()    # they are cleared, so wanted


def test_plan_refusals_and_sizes(L):
    assert L.logra_adapter_plan(NULL, -1, 2, NULL, 0, NULL) == P.ERR_INVALID_ARG
    assert L.logra_adapter_plan(NULL, 4, 0, NULL, 0, NULL) == P.ERR_INVALID_ARG
    assert L.logra_adapter_plan(NULL, 4, 1024, NULL, 0, NULL) == P.ERR_UNSUPPORTED
    assert L.logra_adapter_plan(NULL, 0, 2, NULL, 0, NULL) == P.OK
    assert L.logra_adapter_plan(NULL, 4, 2, NULL, 0, NULL) == P.ERR_INVALID_ARG
    assert P.logra_adapter_plan_size(0, 4) == 0 and P.logra_adapter_plan_size(4, 0) == 0
    assert P.logra_adapter_plan_size(16384, 8) < 1 << 20
    assert P.logra_adapter_ws_size(0, 64, 64, 8, 2) == 0 and P.logra_adapter_ws_size(4, 64, 64, 129, 2) == 0
    # the parts of U and of the gradients, not copies of the rows
    assert P.logra_adapter_ws_size(16384, 4096, 4096, 16, 8) < 32 << 20
    sizes = [P.logra_adapter_ws_size(r, 4096, 4096, 16, 8) for r in (1, 100, 10_000, 1_000_000)]
    assert all(s % 256 == 0 and s > 0 for s in sizes)


def test_forward_workspace_has_no_gradients(L):
    # 96 rows of 64 adapters: four parts of U at most, for rows padded to 32 a group, and not the adapters' gradients
    small, full = (f(96, 4096, 14336, 16, 64) for f in (P.logra_adapter_forward_ws_size, P.logra_adapter_ws_size))
    assert 0 < small <= 4 * (96 + 65 * 32) * 16 * 4 < full and small % 256 == 0
    for bad in ((0, 64, 64, 8, 2), (4, 64, 64, 129, 2), (4, 64, 64, 8, 1024), (4, 1 << 21, 64, 8, 2)):
        assert P.logra_adapter_forward_ws_size(*bad) == 0


def test_dropout_and_loss_refusals(L):
    d = lambda **kw: L.logra_dropout(*{**dict(x=NULL, ld_x=16, dtype=0, rows=2, cols=15, p=0.1, seed=1, off=2, res=NULL,  # noqa: E731
                                              ld_res=16, out=NULL, ld_out=16, st=NULL), **kw}.values())
    for kw in (dict(dtype=2), dict(rows=-1), dict(cols=0), dict(ld_x=12), dict(ld_x=17), dict(ld_out=14), dict(p=1.0),
               dict(p=-1.0), dict()):
        assert d(**kw) == P.ERR_INVALID_ARG
    assert d(rows=1 << 31) == P.ERR_UNSUPPORTED and d(rows=0) == P.OK
    t = lambda **kw: L.logra_token_loss(*{**dict(z=NULL, ld=16, dtype=1, rows=2, vocab=15, t=NULL, w=NULL, loss=NULL,  # noqa: E731
                                                 dz=NULL, ld_d=16, st=NULL), **kw}.values())
    for kw in (dict(dtype=2), dict(rows=-1), dict(vocab=0), dict(ld=8), dict(ld=15), dict(ld=20), dict()):
        assert t(**kw) == P.ERR_INVALID_ARG
    assert t(rows=1 << 31) == P.ERR_UNSUPPORTED and t(vocab=1 << 31, ld=1 << 31) in (P.ERR_UNSUPPORTED, P.ERR_INVALID_ARG)
    assert t(rows=0) == P.OK
