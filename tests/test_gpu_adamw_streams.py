"""The memory of an AdamW plan while steps on other streams are still to run."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("way", ["argument", "number", "current"])
def test_a_plan_that_is_dropped_before_its_step_has_run(way):
    import torch
    import paper_2405_13954_amd as P
    torch.cuda.synchronize()
    tensors = [P.AdamwTensor(*(torch.full((5000,), x, device="cuda") for x in (1.0, 0.5, 0.0, 0.0))) for _ in range(3)]
    step, side = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.cuda.Stream()
    a = torch.randn(4096, 4096, device="cuda")
    plan = P.logra_adamw_plan(tensors, 1)
    at, size = plan.memory.data_ptr(), plan.memory.numel()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(30):                                    # some milliseconds in front of the step
            b = a @ a
    if way == "current":
        with torch.cuda.stream(side):
            P.logra_adamw_step(plan, step, 1e-2)
    else:
        P.logra_adamw_step(plan, step, 1e-2, stream=side if way == "argument" else side.cuda_stream)
    del plan
    busy = not side.query()
    new = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert busy and new.data_ptr() != at, "the plan's memory was handed out before the step had run"
    torch.cuda.synchronize()
    assert int(step) == 1 and all(float((t.param - 0.99).abs().max()) < 1e-6 for t in tensors)
    del new, b
    torch.cuda.synchronize()
    # afterwards it is free again, and a plan on its own stream is as before
    again = P.logra_adamw_plan(tensors, 1)
    P.logra_adamw_step(again, step, 1e-2)
    assert int(step) == 2
