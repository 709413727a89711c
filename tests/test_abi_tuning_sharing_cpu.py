"""Outputs that share memory are refused in calls without rows too, where they are the only memory that is written, and what
an AdamW step reads and writes besides the plan's tensors is apart from these."""
import paper_2405_13954_amd as P
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


def test_a_steps_own_arrays_are_apart_from_the_tensors():
    import torch
    flat = torch.zeros(400)
    t = [P.AdamwTensor(flat[0:20], flat[100:120], flat[20:40], flat[60:80]),
         P.AdamwTensor(flat[200:208], flat[104:112], torch.zeros(8).to(torch.float8_e4m3fn), torch.zeros(8).to(torch.float8_e5m2), flat[300:301],
                       flat[302:303], torch.zeros(8, dtype=torch.bfloat16))]
    arrays = [a for x in t for a in (x.param, x.work, x.m, x.v, x.m_scale, x.v_scale) if a is not None]
    plan = P.AdamwPlan(torch.zeros(4096, dtype=torch.uint8), tuple(t), 4, 0, P._edges(arrays + [x.grad for x in t]), P._edges(arrays))
    step, four = torch.zeros(1, dtype=torch.int64), torch.zeros(4)

    def refused(name, **kw):
        try:
            P.logra_adamw_step(plan, kw.pop("step", step), 1e-3, stream=0, **kw)
        except ValueError as e:
            assert name in str(e) and "share memory" in str(e)
            return True
        except P.LograError as e:                      # the plan is no device memory: past the check
            assert "plan is not" in str(e)
            return False

    parts = {at: flat[at:at + 4] for at in range(0, 396)}
    taken = set(range(0, 40)) | set(range(60, 80)) | set(range(200, 208)) | {300, 302}
    for at, part in parts.items():
        mine = set(range(at, at + 4))
        assert refused("norms", norms=part) == bool(mine & (taken | set(range(100, 120)))), at
        assert refused("lr_scale", lr_scale=part) == bool(mine & taken), at
    for at in range(0, 396, 2):
        here = flat[at:at + 2].view(torch.int64)
        assert refused("step", step=here) == bool({at, at + 1} & (taken | set(range(100, 120)))), at
    assert not refused("norms", norms=four, lr_scale=torch.ones(4))


def test_a_plan_lists_where_its_tensors_are():
    # overlapping stretches are one, neighbours stay two
    import torch
    x, end = torch.zeros(64), 1 << 64
    at = x.data_ptr()
    assert P._edges([]) == P._edges([x[:0]]) == (end,)
    assert P._edges([x[8:16], None, x[0:8], x[12:20], x[13:14]]) == (at, at + 32, at + 32, at + 80, end)
