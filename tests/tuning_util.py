"""Inputs inside guarded buffers and bounds, for the GPU tests of the layer norm, the preference loss and the AdamW step."""
import numpy as np

SENTINEL = 12345.0
U = 2.0 ** -24                       # half a step of fp32, relative
HALF = {"bf16": 2.0 ** -8, "f32": U}   # of an output's one rounding (bf16's is 2^-9 of a binade's top; 2^-8 of the value bounds it)


def dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def mk(g, rows, cols, std, dtype, extra=0, shift=0.0):
    """(device view [rows, cols], float64 copy, the whole buffer): row strides are multiples of 16 bytes, and one row of
    sentinels follows."""
    import torch
    t = torch.from_numpy((g.standard_normal((rows, cols)) * std + shift).astype(np.float32)).to(dt(dtype))
    full = torch.full((rows + 1, -(-cols // 8) * 8 + extra), SENTINEL, dtype=dt(dtype))
    full[:rows, :cols] = t
    full = full.cuda()
    return full[:rows, :cols], t.double().numpy(), full


def room(rows, cols, dtype, extra=0):
    """(view for an output, the whole buffer)."""
    import torch
    full = torch.full((rows + 1, -(-cols // 8) * 8 + extra), SENTINEL, dtype=dt(dtype), device="cuda")
    return full[:rows, :cols], full


def guarded(full, rows, cols):
    keep = full.clone()
    keep[:rows, :cols] = SENTINEL
    assert bool((keep == SENTINEL).all()), "a store outside the rows"


def vector(g, n, std, dtype, shift=0.0):
    import torch
    t = torch.from_numpy((g.standard_normal(n) * std + shift).astype(np.float32)).to(dt(dtype))
    return t.cuda(), t.double().numpy()


def f32(n, fill=SENTINEL):
    import torch
    return torch.full((n,), fill, device="cuda")


def host(t):
    return t.double().cpu().numpy()


def within(got, want, bound, what):
    err = np.abs(got - want)
    bad = ~(err <= bound)
    at = np.argwhere(bad)[:4].tolist()
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} beyond the bound, first at {at}: {err[bad][:4]} > "
                           f"{np.broadcast_to(bound, err.shape)[bad][:4]}")
