"""Refusals and size queries of the layer norm, preference loss and AdamW entry points that need no GPU: every call here
returns from host-side validation.  Addresses are made up; a call that passes the check in question is refused for them
afterwards."""
import ctypes
import random

import pytest

import paper_2405_13954_amd as P

NULL = None
AT = 1 << 40   # an address that no check before the pointers' kinds looks at


@pytest.fixture(scope="module")
def L():
    return P.lib()


def norm_forward(L, **kw):
    a = dict(x=NULL, ld_x=64, dtype=1, rows=4, cols=60, rms=0, eps=1e-5, mask=NULL, gain=NULL, bias=NULL, res=NULL, ld_res=64,
             h=NULL, ld_h=64, y=NULL, ld_y=64, mean=NULL, rstd=NULL, st=NULL)
    return L.logra_layer_norm_forward(*{**a, **kw}.values())


def norm_backward(L, **kw):
    a = dict(h=NULL, ld_h=64, dy=NULL, ld_dy=64, dtype=1, rows=4, cols=60, rms=0, mask=NULL, gain=NULL, mean=NULL, rstd=NULL,
             base=NULL, ld_base=64, dx=NULL, ld_dx=64, dgain=NULL, dbias=NULL, acc=0, ws=NULL, ws_bytes=0, st=NULL)
    return L.logra_layer_norm_backward(*{**a, **kw}.values())


def preference(L, **kw):
    a = dict(z=NULL, ld=64, dtype=1, rows=4, vocab=60, target=NULL, offsets=NULL, pairs=2, ref=NULL, weight=NULL, beta=0.1,
             smoothing=0.0, loss=NULL, logp=NULL, dz=NULL, ld_d=64, ws=NULL, ws_bytes=0, st=NULL)
    return L.logra_preference_loss(*{**a, **kw}.values())


def step(L, **kw):
    a = dict(plan=AT, plan_bytes=1 << 20, groups=2, step=AT * 2, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.0, max_norm=0.0, scale=NULL,
             norms=NULL, seed=0, st=NULL)
    return L.logra_adamw_step(*{**a, **kw}.values())


def shared(status):
    assert status == P.ERR_INVALID_ARG
    return "share memory" in P.logra_last_error()


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), P.ERR_INVALID_ARG), (dict(rows=-1), P.ERR_INVALID_ARG), (dict(cols=0), P.ERR_INVALID_ARG),
    (dict(cols=16385), P.ERR_UNSUPPORTED), (dict(rows=1 << 31), P.ERR_UNSUPPORTED), (dict(), P.ERR_INVALID_ARG)])
def test_norm_sizes(L, change, status):
    assert norm_forward(L, **change) == status and P.logra_last_error()
    assert norm_backward(L, **{**change, "dx": AT}) == status and P.logra_last_error()


def test_norm_refusals(L):
    for kw in (dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(eps=1e-31), dict(rms=1, bias=AT),
               dict(rms=1, mean=AT), dict(ld_x=56), dict(ld_x=62), dict(ld_y=32), dict(res=AT, ld_res=56), dict(h=AT, ld_h=61),
               dict(ld_x=1 << 62)):
        assert norm_forward(L, **kw) == P.ERR_INVALID_ARG, kw
    assert norm_forward(L, rows=0) == P.OK
    for kw in (dict(base=AT), dict(rms=1, dbias=AT), dict(rms=1, dgain=AT, mean=AT), dict(dx=AT, ld_h=56), dict(dx=AT, ld_dy=62),
               dict(dx=AT, ld_dx=56), dict(dx=AT, base=AT, ld_base=32), dict(dx=AT)):
        assert norm_backward(L, **kw) == P.ERR_INVALID_ARG, kw
    assert norm_backward(L) == P.OK                          # no gradient is wanted
    assert norm_backward(L, rows=0, dx=AT) == P.OK
    assert P.logra_layer_norm_ws_size(0, 64) == 0 and P.logra_layer_norm_ws_size(4, 16385) == 0
    sizes = [P.logra_layer_norm_ws_size(r, 4096) for r in (1, 100, 16384, 1 << 30)]
    assert sizes == sorted(sizes) and all(s % 256 == 0 and 0 < s <= 64 << 20 for s in sizes)


def test_norm_operands_are_in_place_or_apart(L):
    far = dict(x=AT, y=AT * 2)
    assert not shared(norm_forward(L, **far))
    assert not shared(norm_forward(L, x=AT, y=AT)) and not shared(norm_forward(L, x=AT, y=AT, res=AT * 2, h=AT * 2))
    assert not shared(norm_forward(L, x=AT, y=AT * 2, res=AT * 3, h=AT))
    assert shared(norm_forward(L, x=AT, y=AT, res=AT * 2, h=AT))              # two outputs in one place
    assert shared(norm_forward(L, x=AT, y=AT + 128)) and shared(norm_forward(L, x=AT, y=AT, ld_y=128))
    assert shared(norm_forward(L, **far, res=AT * 2 + 16)) and shared(norm_forward(L, **far, gain=AT * 2 + 64))
    assert shared(norm_forward(L, **far, mean=AT + 4)) and shared(norm_forward(L, **far, mean=AT * 3, rstd=AT * 3 + 12))
    assert shared(norm_forward(L, **far, mask=AT * 3 + 1, rstd=AT * 3))
    assert not shared(norm_forward(L, **far, mean=AT * 3, rstd=AT * 3 + 16))
    far = dict(h=AT, dy=AT * 2)
    for name in ("h", "dy"):
        assert not shared(norm_backward(L, **far, dx=far[name])) and shared(norm_backward(L, **far, dx=far[name] + 16))
        assert shared(norm_backward(L, **far, dx=far[name], ld_dx=128)) and shared(norm_backward(L, **far, dgain=far[name] + 64))
    assert not shared(norm_backward(L, **far, dx=AT * 3, base=AT * 3)) and shared(norm_backward(L, **far, dx=AT * 3, base=AT * 3 + 128))
    assert shared(norm_backward(L, **far, dgain=AT * 3, dbias=AT * 3 + 236)) and not shared(norm_backward(L, **far, dgain=AT * 3, dbias=AT * 3 + 240))
    assert shared(norm_backward(L, **far, dgain=AT * 3, mean=AT * 3 + 236)) and shared(norm_backward(L, **far, dx=AT * 3, rstd=AT * 3))
    assert shared(norm_backward(L, **far, dgain=AT * 3, ws=AT * 2 - 4, ws_bytes=256))


def test_preference_refusals(L):
    for kw in (dict(dtype=2), dict(rows=-1), dict(vocab=0), dict(pairs=-1), dict(beta=INF), dict(beta=NAN), dict(smoothing=-0.1),
               dict(smoothing=1.1), dict(smoothing=NAN), dict(ld=56), dict(ld=60), dict(dz=AT, ld_d=56), dict(pairs=0, dz=AT), dict()):
        assert preference(L, **kw) == P.ERR_INVALID_ARG, kw
    assert preference(L, rows=1 << 31) == P.ERR_UNSUPPORTED and preference(L, pairs=(1 << 29) + 1) == P.ERR_UNSUPPORTED
    assert preference(L, vocab=(1 << 30) + 1) == P.ERR_UNSUPPORTED
    assert preference(L, pairs=0) == P.OK and preference(L, pairs=0, rows=0) == P.OK
    assert P.logra_preference_loss_ws_size(0, 2) == 0 and P.logra_preference_loss_ws_size(4, 0) == 0
    # a few numbers for each token, nothing the size of its logits
    assert 0 < P.logra_preference_loss_ws_size(2048, 8) <= 2048 * 256
    assert P.logra_preference_loss_ws_size(1000, 8) % 256 == 0


def test_preference_operands_are_in_place_or_apart(L):
    far = dict(z=AT, target=AT * 2, offsets=AT * 3, logp=AT * 4)
    assert not shared(preference(L, **far, dz=AT)) and not shared(preference(L, **far, dz=AT * 5))
    assert shared(preference(L, **far, dz=AT, ld_d=72)) and shared(preference(L, **far, dz=AT + 128))
    assert shared(preference(L, **far, dz=AT * 2 + 16)) and shared(preference(L, **far, loss=AT * 4 + 12))
    assert shared(preference(L, **far, ref=AT * 4 + 12)) and shared(preference(L, **far, weight=AT * 4 + 12))
    assert shared(preference(L, **far, loss=AT * 3 + 36)) and not shared(preference(L, **far, loss=AT * 3 + 40))
    assert shared(preference(L, **far, ws=AT * 4 - 256, ws_bytes=260)) and not shared(preference(L, **far, ws=AT * 4 - 256, ws_bytes=256))


def tensor(**kw):
    return P.AdamwDesc(**{**dict(param=AT, work=None, grad=AT * 2, m=AT * 3, v=AT * 4, m_scale=None, v_scale=None, slice=100, slices=2,
                                 first_group=0, decay=1), **kw})


def plan(L, tensors, groups, plan=AT * 8, plan_bytes=1 << 30):
    return L.logra_adamw_plan((P.AdamwDesc * max(1, len(tensors)))(*tensors), len(tensors), groups, plan, plan_bytes, NULL)


def test_plan_refusals(L):
    for t in (tensor(slice=-1), tensor(slices=-1), tensor(first_group=-1), tensor(first_group=1), tensor(slices=3), tensor(m_scale=AT),
              tensor(v_scale=AT), tensor()):                            # the last: no device memory
        assert plan(L, [t], 2) == P.ERR_INVALID_ARG
    assert plan(L, [tensor(slice=1 << 31)], 2) == P.ERR_UNSUPPORTED
    assert plan(L, [tensor()], 0) == P.ERR_INVALID_ARG and plan(L, [tensor()], 65537) == P.ERR_UNSUPPORTED
    assert L.logra_adamw_plan(None, 1, 2, AT, 1 << 20, NULL) == P.ERR_INVALID_ARG
    assert L.logra_adamw_plan(None, -1, 2, AT, 1 << 20, NULL) == P.ERR_INVALID_ARG
    assert plan(L, [tensor()], 2, plan=None) == P.ERR_WORKSPACE and plan(L, [tensor()], 2, plan_bytes=512) == P.ERR_WORKSPACE
    # 2^31 - 1 slices of 2^31 - 1 elements: more chunks than a plan holds
    assert plan(L, [tensor(slice=(1 << 31) - 1, slices=2)], 2, plan_bytes=1 << 20) == P.ERR_WORKSPACE
    assert plan(L, [tensor(slice=(1 << 31) - 1, slices=65536)] * 64, 65536) == P.ERR_UNSUPPORTED


def test_plan_sizes(L):
    size = lambda ts, n: int(L.logra_adamw_plan_size((P.AdamwDesc * max(1, len(ts)))(*ts), len(ts), n))  # noqa: E731
    assert size([tensor()], 0) == 0 and size([tensor()], 65537) == 0 and size([tensor(slice=-1)], 2) == 0
    assert 0 < size([], 1) < 2048
    # for every 2,048 elements of a slice a hundred bytes, not copies of them
    one = size([tensor(slice=1 << 20, slices=8)], 8)
    assert 8 * 512 * 64 <= one <= 8 * 512 * 128 and one % 256 == 0
    assert size([tensor(slice=1, slices=8)], 8) == size([tensor(slice=2048, slices=8)], 8) < size([tensor(slice=2049, slices=8)], 8)


def test_step_refusals(L):
    for kw in (dict(groups=0), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=NAN), dict(eps=0.0), dict(eps=INF), dict(lr=INF),
               dict(lr=NAN), dict(wd=-1.0), dict(wd=INF), dict(max_norm=-1.0), dict(max_norm=NAN), dict()):
        assert step(L, **kw) == P.ERR_INVALID_ARG, kw
    assert step(L, groups=65537) == P.ERR_UNSUPPORTED
    assert step(L, plan=None) == P.ERR_WORKSPACE and step(L, plan_bytes=256) == P.ERR_WORKSPACE
    assert shared(step(L, step=AT + 8)) and shared(step(L, norms=AT + 8)) and shared(step(L, scale=AT + 8))
    assert shared(step(L, norms=AT * 2 + 4)) and shared(step(L, norms=AT * 3, scale=AT * 3 + 4))
    assert not shared(step(L, norms=AT * 3, scale=AT * 3 + 8))


def test_python_checks():
    import torch
    x, y, f = torch.zeros(4, 16), torch.zeros(4, 16), torch.zeros(16)
    with pytest.raises(ValueError):
        P.logra_layer_norm_forward(x, torch.zeros(4, 8))
    with pytest.raises(ValueError):
        P.logra_layer_norm_forward(x, y, gain=torch.zeros(8))
    with pytest.raises(ValueError):
        P.logra_layer_norm_forward(x, y, gain=f.to(torch.bfloat16))
    with pytest.raises(ValueError):
        P.logra_layer_norm_forward(x, y, mask=torch.zeros(4, dtype=torch.bool))
    with pytest.raises(ValueError):
        P.logra_layer_norm_backward(x, y, torch.zeros(3))
    with pytest.raises(ValueError):
        P.logra_preference_loss(x, torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int64), torch.zeros(2))
    with pytest.raises(ValueError):
        P.logra_adamw_plan([P.AdamwTensor(f, f, f.to(torch.float8_e4m3fn), f.to(torch.float8_e5m2))], 1)   # no scales
    with pytest.raises(ValueError):
        P.logra_adamw_plan([P.AdamwTensor(f, f, f, f, f[:1], f[:1])], 1)                                   # scales of fp32 states
    with pytest.raises(ValueError):
        P.logra_adamw_plan([P.AdamwTensor(f, f, f, f, slices=3)], 1)


def test_the_descriptor_is_the_headers(L):
    assert ctypes.sizeof(P.AdamwDesc) == 80 and P.AdamwDesc.slice.offset == 56 and P.AdamwDesc.decay.offset == 72


def test_norm_sharing_is_that_of_the_bytes(L):
    # the answer against the sets of bytes, for an output that is neither in place nor plainly apart
    g = random.Random(7)
    seen = {True: 0, False: 0}
    for _ in range(1500):
        rows, cols = g.randint(1, 5), g.randint(1, 30)
        least = -(-cols // 8)
        ld_h, ld_d = (8 * (least + g.choice((0, 1, 5))) for _ in range(2))
        shift = 2 * g.randint(-2 * ld_h * rows, 2 * ld_h * rows)
        if shift == 0:
            continue
        a = {r * 2 * ld_h + b for r in range(rows) for b in range(2 * cols)}
        b = {shift + r * 2 * ld_d + b for r in range(rows) for b in range(2 * cols)}
        want = bool(a & b)
        got = shared(norm_backward(L, rows=rows, cols=cols, h=AT, ld_h=ld_h, dy=AT * 2, dx=AT + shift, ld_dx=ld_d, ld_dy=8 * least))
        assert got == want, (rows, cols, ld_h, ld_d, shift)
        seen[want] += 1
    assert min(seen.values()) > 200
