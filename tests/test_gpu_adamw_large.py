"""AdamW steps whose groups have more chunks of 2,048 elements than the sums of a launch are added in at once, and plans on either
side of the limit between the two ways to a group's factors, against float64 on the device.  Bounds as in test_gpu_adamw.py.
"""
import math

import pytest

from tuning_util import U

pytestmark = pytest.mark.gpu
CHUNK = 2048


def close(got, want, bound, what):
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), f"{what}: {float((err - bound).max()):.3e} beyond the bound at {int((err - bound).argmax())}"


# 1,024 chunks: the last plan whose step has no launch of its own for the factors; 2,348: 300 more than are added at once
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("chunks", [1023, 1024, 1025, 2348, 4400])
def test_a_group_of_many_chunks(chunks, bits):
    import torch
    import paper_2405_13954_amd as P
    print("[adamw, many chunks]", chunks, bits, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(chunks)
    normal = lambda n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    tensors, grads = [], []
    for i, n in enumerate((700, (chunks - 3) * CHUNK - 5, 2 * CHUNK)):      # the first in group 0, the others in group 1
        grad = normal(n) * 1e-3
        grad[min(2048, chunks // 2) * CHUNK:] *= 10.0                      # what a lost chunk would take from the norm shows
        m, v = normal(n) * 1e-3, (normal(n) * 1e-3).square()
        scales = {}
        if bits == 8:
            blocks = -(-n // P.ADAMW_BLOCK)
            scales = dict(m_scale=torch.full((blocks,), 2.0 ** -16, device="cuda"), v_scale=torch.full((blocks,), 2.0 ** -30, device="cuda"))
            m, v = (m * 2.0 ** 16).clamp(-448, 448).to(torch.float8_e4m3fn), (v * 2.0 ** 30).clamp(max=57344).to(torch.float8_e5m2)
        grads.append(grad)
        tensors.append(P.AdamwTensor(normal(n) * 0.1, grad, m, v, first_group=min(i, 1), work=torch.empty(n, dtype=torch.bfloat16, device="cuda"),
                                     **scales))
    square = [float(g.double().square().sum()) for g in grads]
    norm = [math.sqrt(square[0]), math.sqrt(square[1] + square[2])]
    plan = P.logra_adamw_plan(tensors, 2)
    wide = lambda t, n: t.float().double() if n is None else t.float().double() * n.double().repeat_interleave(P.ADAMW_BLOCK)[:t.numel()]  # noqa: E731
    before = [(t.param.double().clone(), wide(t.m, t.m_scale).clone(), wide(t.v, t.v_scale).clone()) for t in tensors]
    step, norms, most = torch.full((1,), 4, dtype=torch.int64, device="cuda"), torch.empty(2, device="cuda"), norm[1] / 3
    lr, b1, b2, eps, wd = 1e-2, 0.9, 0.95, 1e-6, 0.1
    P.logra_adamw_step(plan, step, lr, beta1=b1, beta2=b2, eps=eps, weight_decay=wd, max_norm=most, norms=norms, seed=9)
    assert int(step) == 5
    assert all(abs(float(a) - b) <= 2 * U * b for a, b in zip(norms, norm)), (norms.tolist(), norm)
    for i, (t, g, (p, m, v)) in enumerate(zip(tensors, grads, before)):
        clip = min(1.0, most / norm[min(i, 1)])
        cg = clip * g.double()
        m2, v2 = b1 * m + (1 - b1) * cg, b2 * v + (1 - b2) * cg * cg
        em, ev = 4 * U * (b1 * m.abs() + (1 - b1) * cg.abs()) + 1e-44, 6 * U * v2 + 1e-44
        if bits == 32:
            close(t.m, m2, em, f"m of tensor {i}")
            close(t.v, v2, ev, f"v of tensor {i}")
        move = lr / (1 - b1 ** 5) / ((v2 / (1 - b2 ** 5)).sqrt() + eps)
        bound = move * em + move * m2.abs() * (0.5 * ev / (v2 + 1e-300) + 8 * U) + 3 * U * (p.abs() + move * m2.abs())
        close(t.param, p * (1 - lr * wd) - move * m2, bound, f"param of tensor {i}")
        assert torch.equal(t.work, t.param.to(torch.bfloat16))


def test_a_group_of_many_chunks_that_are_not_finite():
    # a gradient that is not finite in the last chunk, which the second batch of sums holds: its group stays as it is
    import torch
    import paper_2405_13954_amd as P
    n = 2349 * CHUNK
    param, grad, m, v = torch.ones(n, device="cuda"), torch.ones(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    grad[-1] = float("inf")
    plan, step, norms = P.logra_adamw_plan([P.AdamwTensor(param, grad, m, v)], 1), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty(1, device="cuda")
    P.logra_adamw_step(plan, step, 1e-2, max_norm=1.0, norms=norms)
    assert torch.isinf(norms).all() and bool((param == 1).all()) and not m.any() and not v.any() and int(step) == 1
