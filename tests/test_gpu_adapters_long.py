"""Adapters where a call takes the rarer turns of the kernels: runs of the gradient longer than the 32 blocks whose rows
are looked up together, du in as many parts as there can be, stores beyond 32-bit offsets, the most rows and adapters."""
import numpy as np
import pytest

from test_gpu_adapters import _case, _check_backward, _check_forward, _forward, _plan
from test_gpu_adapters_large import test_forward_and_backward as check

pytestmark = pytest.mark.gpu


# 2,500 rows are about 80 blocks of 32; 512 slices of 256 columns beside the other side's leave one run of them all.
# One adapter goes on from chunk to chunk, three and 40 change inside them.
@pytest.mark.parametrize("shape,dtype,p", [
    ((2500, 64, 131072, 9, 3), "bf16", 0.0), ((2500, 64, 131072, 16, 1), "f32", 0.0), ((2500, 131072, 64, 16, 3), "bf16", 0.1),
    ((2500, 131072, 64, 12, 3), "f32", 0.1), ((2500, 64, 131072, 40, 2), "bf16", 0.0), ((2500, 131072, 64, 60, 40), "f32", 0.0),
    ((2500, 131072, 64, 100, 2), "bf16", 0.1)])
def test_runs_longer_than_a_chunk(shape, dtype, p):
    import torch
    check(shape, dtype, p)
    torch.cuda.empty_cache()


# 300 rows of 4096 outputs: the long axis in four ranges
@pytest.mark.parametrize("p", [0.0, 0.1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(300, 264, 4096, 9, 3), (300, 4096, 4096, 16, 2), (40, 136, 8192, 4, 1)])
def test_four_parts_of_du(shape, dtype, p):
    check(shape, dtype, p)


def test_stores_beyond_32_bits():
    # 40 rows of y and dx at a stride of 2^28 bytes or more: byte offsets to 2^33, in place and apart
    import torch
    import paper_2405_13954_amd as P
    for dtype, dt, elements in (("bf16", torch.bfloat16, 40 << 27), ("f32", torch.float32, 20 << 27)):
        c = _case(21, 40, 64, 32, 16, 2, dtype)
        wide = torch.empty(elements, dtype=dt, device="cuda").view(40, -1)
        plan = _plan(c)
        y, u, _ = _forward(c, plan)
        P.logra_adapter_forward(c["x"], c["a"], c["b"], plan, wide[:, 64:96], base=c["base"], scale=c["scale"])
        assert torch.equal(wide[:, 64:96], y)
        da, db = torch.empty(2, 16, 64, device="cuda"), torch.empty(2, 16, 32, device="cuda")
        dx = torch.empty(40, 64, dtype=dt, device="cuda")
        for out in (dx, wide[:, 128:192]):
            P.logra_adapter_backward(c["x"], c["dy"], c["a"], c["b"], plan, u, da, db, dx=out, base=c["back"], scale=c["scale"])
        assert torch.equal(wide[:, 128:192], dx)
        base, back = wide[:, 256:288], wide[:, 512:576]
        base.copy_(c["base"])
        back.copy_(c["back"])
        c["base"], c["back"] = base, back
        _check_forward(c, inplace=True)
        _check_backward(c, inplace=True)
        del wide, base, back, c


def test_most_rows_and_adapters():
    # 2^24 rows in any order of 1,023 adapters, small integers: every sum is exact, whatever its order
    import torch
    import paper_2405_13954_amd as P
    rows, n = 1 << 24, 1023
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    small = lambda *s: torch.randint(-1, 2, s, generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
    ids = torch.randint(-1, n + 1, (rows,), generator=g, device="cuda", dtype=torch.int32)
    live = (ids >= 0) & (ids < n)
    at = torch.where(live, ids, n).long()            # group n: none
    x, dy, a, b = small(rows, 8), small(rows, 8), small(n, 1, 8), small(n, 1, 8)
    bf = lambda t: t.to(torch.bfloat16)  # noqa: E731
    print("[adapters] 2^24 rows", flush=True)
    plan = P.logra_adapter_plan(ids, n)
    y, u, dx = (torch.empty(rows, 8, device="cuda", dtype=torch.bfloat16), torch.empty(rows, 1, device="cuda"),
                torch.empty(rows, 8, device="cuda", dtype=torch.bfloat16))
    da, db = torch.empty(n, 1, 8, device="cuda"), torch.empty(n, 1, 8, device="cuda")
    P.logra_adapter_forward(bf(x), bf(a), bf(b), plan, y, u=u)
    P.logra_adapter_backward(bf(x), bf(dy), bf(a), bf(b), plan, u, da, db, dx=dx)
    aa, bb = (torch.cat([t[:, 0].float(), torch.zeros(1, 8, device="cuda")])[at] for t in (a, b))
    want_u, du = (aa * x).sum(1, keepdim=True), (bb * dy).sum(1, keepdim=True)
    assert torch.equal(u, want_u) and torch.equal(y.float(), want_u * bb) and torch.equal(dx.float(), du * aa)
    order = at.argsort()
    ends = torch.searchsorted(at[order], torch.arange(n, device="cuda"), right=True)
    assert bool((ends > 0).all())
    for got, left, right in ((da, du, x), (db, want_u, dy)):
        sums = (left * right).double()[order].cumsum(0)[ends - 1]          # a group's rows up to and with its last
        want = torch.cat([sums[:1], sums[1:] - sums[:-1]])
        assert torch.equal(got[:, 0].double(), want)
