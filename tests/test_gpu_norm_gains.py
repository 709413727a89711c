"""Layer norm under the gains and biases of several models of an odd width, one behind the other, as a step leaves them: the same
bits as under a copy of each at an aligned place."""
import pytest

from tuning_util import dt, f32

pytestmark = pytest.mark.gpu


def buffer(g, rows, cols, dtype):
    import torch
    full = torch.full((rows, -(-cols // 8) * 8 + 8), float("nan"), dtype=dt(dtype), device="cuda")
    full[:, :cols] = torch.randn(rows, cols, generator=g, device="cuda")
    return full[:, :cols]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(6, 1), (6, 77), (6, 1001), (6, 8203), (1030, 77), (1030, 1001), (1030, 4109), (1030, 12299)])
def test_gains_of_several_models(rows, cols, dtype):
    import torch
    import paper_2405_13954_amd as P
    print("[norm, gains]", rows, cols, dtype, flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    x, dy = buffer(g, rows, cols, dtype), buffer(g, rows, cols, dtype)
    # what lies before the first gain and behind the last is not read: NaN
    m, flat = 5, torch.full((5 * cols * 2 + 2,), float("nan"), dtype=dt(dtype), device="cuda")
    gains, biases = flat[1:1 + m * cols].view(m, cols), flat[1 + m * cols:1 + 2 * m * cols].view(m, cols)
    gains.copy_(1 + 0.3 * torch.randn(m, cols, generator=g, device="cuda"))
    biases.copy_(0.3 * torch.randn(m, cols, generator=g, device="cuda"))
    for s in (0, 1, 2, m - 1):
        for rms in (False, True):
            out = []
            for gain, bias in ((gains[s], biases[s]), (gains[s].clone(), biases[s].clone())):
                y, dx, mean, rstd, dgain = buffer(g, rows, cols, dtype), buffer(g, rows, cols, dtype), f32(rows), f32(rows), f32(cols)
                stat = None if rms else mean
                P.logra_layer_norm_forward(x, y, gain=gain, bias=None if rms else bias, rms=rms, mean=stat, rstd=rstd)
                P.logra_layer_norm_backward(x, dy, rstd, mean=stat, gain=gain, rms=rms, dx=dx, dgain=dgain)
                out.append((y, dx, rstd, dgain))
            assert all(torch.equal(a, b) and bool(torch.isfinite(a).all()) for a, b in zip(*out)), (s, rms)


def test_the_copies_that_a_step_writes():
    import torch
    import paper_2405_13954_amd as P
    m, cols = 3, 77
    g = torch.Generator(device="cuda").manual_seed(1)
    param, grad = torch.ones(m, cols, device="cuda"), torch.randn(m, cols, generator=g, device="cuda")
    work = torch.zeros(m, cols, dtype=torch.bfloat16, device="cuda")
    plan = P.logra_adamw_plan([P.AdamwTensor(param, grad, torch.zeros_like(param), torch.zeros_like(param), work=work, slices=m)], m)
    P.logra_adamw_step(plan, torch.zeros(1, dtype=torch.int64, device="cuda"), 0.1)
    x = buffer(g, 12, cols, "bf16")
    y, want = buffer(g, 12, cols, "bf16"), buffer(g, 12, cols, "bf16")
    for s in range(m):
        part = slice(4 * s, 4 * s + 4)
        P.logra_layer_norm_forward(x[part], y[part], gain=work[s], rms=True)
        P.logra_layer_norm_forward(x[part], want[part], gain=param[s].to(torch.bfloat16), rms=True)
    assert torch.equal(y, want) and bool((work != 1).any())


def test_a_gain_at_no_elements_place():
    import torch
    import paper_2405_13954_amd as P
    x, raw = torch.randn(4, 16, device="cuda"), torch.zeros(68, dtype=torch.uint8, device="cuda")
    args = [x.data_ptr(), 16, 0, 4, 16, 1, 1e-5, None, raw.data_ptr() + 2, None, None, 0, None, 0, torch.empty_like(x).data_ptr(), 16, None, None, None]
    assert P.lib().logra_layer_norm_forward(*args) == P.ERR_INVALID_ARG and "aligned" in P.logra_last_error()
