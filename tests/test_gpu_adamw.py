"""The AdamW step against the float64 oracle.

8-bit states and their scales have to be equal: the kernel forms them in float64, where only a value within 2^-50 of the
boundary that its random bits set could differ.  In fp32 m and v are within 4 and 6 u (u = 2^-24) of their terms' magnitudes (two
products, a sum, the clipped gradient's rounding, once or squared).  The move lr mhat / (sqrt(vhat) + eps) carries m's bound,
half of v's and 8 roundings (clip, rate, root, product, square root, sum, quotient); param its own two.
"""
import numpy as np
import pytest

from oracle import tuning as O
from tuning_util import U, host, within

pytestmark = pytest.mark.gpu
GUARD = 7   # elements of sentinels around every array, so that none begins at a multiple of 16 bytes


def _inside(a, dtype):
    """The values of `a` in the middle of a longer buffer of sentinels: (view, buffer)."""
    import torch
    src = torch.from_numpy(np.asarray(a, dtype=np.float64).reshape(-1))
    full = torch.full((len(src) + 2 * GUARD,), 96.0, dtype=torch.float64)
    full[GUARD:GUARD + len(src)] = src
    full = full.to(torch.float32).to(dtype).cuda()
    return full[GUARD:GUARD + len(src)], full


class Model:
    """Tensors on the device, each guarded, and their float64 values."""

    def __init__(self, g, shapes, bits, work=True, decay=None, zero_state=False):
        import torch
        import paper_2405_13954_amd as P
        self.host, self.dev, self.full, self.tensors = [], [], [], []
        for i, (slices, n, first) in enumerate(shapes):
            b = bits[i] if isinstance(bits, (list, tuple)) else bits
            blocks = -(-n // O.BLOCK)
            one = dict(param=g.standard_normal((slices, n)) * 0.1, grad=g.standard_normal((slices, n)) * 10.0 ** g.uniform(-6, 0, (slices, n)))
            m, v = g.standard_normal((slices, n)) * 1e-2, g.standard_normal((slices, n)) ** 2 * 1e-3
            if zero_state:
                m, v = m * 0, v * 0
            if b == 8:
                one["m_scale"], one["v_scale"] = np.full((slices, blocks), 2.0 ** -12), np.full((slices, blocks), 2.0 ** -24)
                if zero_state:
                    one["m_scale"], one["v_scale"] = one["m_scale"] * 0, one["v_scale"] * 0
                one["m"], one["v"] = np.clip(m * 2.0 ** 12, -448, 448), np.clip(v * 2.0 ** 24, 0, 57344)
            else:
                one["m"], one["v"] = m, v
            types = dict(param=torch.float32, grad=torch.float32, m_scale=torch.float32, v_scale=torch.float32,
                         m=torch.float8_e4m3fn if b == 8 else torch.float32, v=torch.float8_e5m2 if b == 8 else torch.float32)
            pairs = {k: _inside(x, types[k]) for k, x in one.items()}
            if work:
                pairs["work"] = _inside(np.zeros(slices * n), torch.bfloat16)
            self.dev.append({k: p[0] for k, p in pairs.items()})
            self.full.append({k: p[1] for k, p in pairs.items()})
            dec = decay[i] if decay else i % 3 != 2
            self.host.append(dict(first_group=first, decay=dec, bits=b, slices=slices))
            self.tensors.append(P.AdamwTensor(**self.dev[-1], slices=slices, first_group=first, decay=dec))

    def values(self):
        """What the device holds, as the oracle takes it."""
        out = []
        for h, d in zip(self.host, self.dev):
            s = h["slices"]
            x = {k: host(t).reshape(s, -1) for k, t in d.items() if k != "work"}
            if h["bits"] == 8:
                n = x["param"].shape[1]
                for k in ("m", "v"):
                    x[k] = x[k] * np.repeat(x[k + "_scale"], O.BLOCK, axis=1)[:, :n]
            out.append({**h, **x})
        return out

    def guards(self):
        for f in self.full:
            for k, t in f.items():
                edge = t.float()
                assert bool((edge[:GUARD] == 96).all()) and bool((edge[-GUARD:] == 96).all()), f"a store outside {k}"


def check_steps(g, shapes, bits, n_groups, steps=3, work=True, zero_state=False, decay=None, **hyper):
    import torch
    import paper_2405_13954_amd as P
    print("[adamw]", shapes, bits, hyper, flush=True)
    model = Model(g, shapes, bits, work, decay, zero_state)
    plan = P.logra_adamw_plan(model.tensors, n_groups)
    lr, b1, b2, eps = 1e-2, 0.9, 0.95, hyper.pop("eps", 1e-6)
    wd, max_norm, seed = hyper.pop("weight_decay", 0.1), hyper.pop("max_norm", 0.0), hyper.pop("seed", 0xFEDCBA9876543210)
    scale64 = np.array([0.5, 2.0, 0.0, 1.25])[np.arange(n_groups) % 4] if hyper.pop("lr_scale", True) else None
    scale = None if scale64 is None else torch.from_numpy(scale64).float().cuda()
    norms = torch.full((n_groups + 1,), 7.0, device="cuda") if hyper.pop("norms", True) else None
    at = hyper.pop("at", 0)
    assert not hyper
    step = torch.tensor([at, 99], device="cuda")
    for k in range(steps):
        before = model.values()
        want, want_norms = O.adamw_step(before, n_groups, at + k, lr, b1, b2, eps, wd, max_norm, scale64, norms is not None, seed)
        P.logra_adamw_step(plan, step[:1], lr, beta1=b1, beta2=b2, eps=eps, weight_decay=wd, max_norm=max_norm, lr_scale=scale,
                           norms=None if norms is None else norms[:n_groups], seed=seed)
        assert step.tolist() == [at + k + 1, 99]
        got = model.values()
        if norms is not None:
            within(host(norms[:n_groups]), want_norms, 2 * U * want_norms, "norms")
            assert norms[n_groups] == 7
        for i, (x, y, z) in enumerate(zip(before, got, want)):
            s = x["first_group"] + np.arange(x["slices"])
            c = np.where((want_norms > max_norm) & (max_norm > 0), max_norm / np.maximum(want_norms, 1e-300), 1.0)[s][:, None]
            cg = np.abs(c * x["grad"])
            rate = lr * (np.ones(n_groups) if scale64 is None else scale64)[s][:, None]
            if x["bits"] == 8:
                for name in ("m_scale", "v_scale", "m", "v"):
                    assert np.array_equal(y[name], z[name]), f"{name} of tensor {i}, step {k}"
            m, v = b1 * x["m"] + (1 - b1) * c * x["grad"], b2 * x["v"] + (1 - b2) * cg ** 2
            em, ev = 4 * U * (b1 * np.abs(x["m"]) + (1 - b1) * cg) + 1e-44, 6 * U * v + 1e-44
            if x["bits"] == 32:
                within(y["m"], z["m"], em, f"m of tensor {i}")
                within(y["v"], z["v"], ev, f"v of tensor {i}")
            t = at + k + 1
            denom = np.sqrt(v / (1 - b2 ** t)) + eps
            move = rate / (1 - b1 ** t) / denom
            bound = move * em + move * np.abs(m) * (0.5 * ev / (v + 1e-300) + 8 * U) + 3 * U * (np.abs(x["param"]) + move * np.abs(m))
            within(y["param"], z["param"], bound, f"param of tensor {i}")
            if work:
                assert torch.equal(model.dev[i]["work"], model.dev[i]["param"].to(torch.bfloat16)), f"work of tensor {i}"
        model.guards()
    return model


SMALL = [(1, 1, 0), (3, 7, 0), (2, 256, 1), (1, 1001, 2), (4, 300, 0), (1, 2048, 3), (2, 4100, 1)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("max_norm", [0.0, 1.0])
def test_steps(bits, max_norm):
    check_steps(np.random.default_rng(1), SMALL, bits, 4, max_norm=max_norm)


def test_scales_of_any_value_and_no_momentum():
    import torch
    import paper_2405_13954_amd as P
    for b1, b2 in ((0.9, 0.999), (0.0, 0.0)):
        model = Model(np.random.default_rng(14), [(2, 700, 0)], 8)
        for k in ("m_scale", "v_scale"):                       # a checkpoint's scales need not be powers of two
            model.dev[0][k].copy_(torch.rand(6, device="cuda") * 0.01)
        before = model.values()
        step = torch.full((1,), 3, dtype=torch.int64, device="cuda")
        P.logra_adamw_step(P.logra_adamw_plan(model.tensors, 2), step, 1e-3, beta1=b1, beta2=b2, seed=1)
        got, (want,) = model.values()[0], O.adamw_step(before, 2, 3, 1e-3, b1, b2, seed=1)[0]
        for k in ("m", "v", "m_scale", "v_scale"):
            assert np.array_equal(got[k], want[k]), k
        within(got["param"], want["param"], 16 * U * (np.abs(want["param"]) + np.abs(want["param"] - before[0]["param"])), "param")
        model.guards()


def test_mixed_states_and_no_work():
    check_steps(np.random.default_rng(2), SMALL, [8, 32, 32, 8, 8, 32, 8], 5, work=False, max_norm=0.5, at=1000)


@pytest.mark.parametrize("bits", [32, 8])
def test_from_zero_states(bits):
    check_steps(np.random.default_rng(3), [(2, 515, 0), (1, 64, 1)], bits, 2, zero_state=True, norms=False, lr_scale=False)


@pytest.mark.parametrize("bits", [32, 8])
def test_without_norms_decay_or_scales(bits):
    check_steps(np.random.default_rng(4), SMALL, bits, 4, steps=1, norms=False, lr_scale=False, weight_decay=0.0, seed=3, at=1 << 33)


def test_a_tensor_of_many_chunks_and_many_groups():
    check_steps(np.random.default_rng(5), [(37, 4096 + 8, 0), (1, 70001, 36)], 32, 40, steps=1, max_norm=3.0)
    check_steps(np.random.default_rng(6), [(9, 2056, 2)], 8, 11, steps=1, max_norm=3.0)


def test_a_plan_of_thousands_of_chunks():
    check_steps(np.random.default_rng(12), [(2, (1 << 20) + 5, 0), (1, 300, 1), (3, 70, 0)], 32, 4, steps=2, max_norm=400.0)


def test_the_ways_to_a_groups_factors_agree():
    # a plan in more memory than it needs counts as one of many chunks, whose groups get a launch of their own
    import ctypes
    import torch
    import paper_2405_13954_amd as P
    shapes = [(3, 5000, 1), (1, 777, 0), (2, 256, 2)]
    for bits in (32, 8):
        runs = []
        for wide in (False, True):
            model = Model(np.random.default_rng(13), shapes, bits)
            plan = P.logra_adamw_plan(model.tensors, 5)
            if wide:
                descs = (P.AdamwDesc * len(model.tensors))(*[P._adamw_desc(t, i) for i, t in enumerate(model.tensors)])
                memory = torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
                stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
                assert P.lib().logra_adamw_plan(descs, len(descs), 5, memory.data_ptr(), memory.numel(), stream) == P.OK
                plan = plan._replace(memory=memory)
            step, norms = torch.full((1,), 6, dtype=torch.int64, device="cuda"), torch.full((5,), 9.0, device="cuda")
            scale = torch.tensor([1.0, 0.5, 2.0, 0.25, 3.0], device="cuda")
            for _ in range(3):
                P.logra_adamw_step(plan, step, 1e-2, max_norm=2.0, lr_scale=scale, norms=norms, weight_decay=0.1, seed=3)
            assert int(step) == 9 and norms[4] == 0            # (no tensor of group 4)
            runs.append([t.clone().view(torch.uint8) for d in model.dev for t in d.values()] + [norms.view(torch.uint8)])
        assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_the_plain_adam_of_small_gradients():
    # gradients of 1e-20: v is below the smallest normal fp32 number, and the move is that of eps
    import torch
    import paper_2405_13954_amd as P
    for bits in (32, 8):
        g = np.random.default_rng(7)
        model = Model(g, [(1, 300, 0)], bits, zero_state=True, decay=[False])
        model.dev[0]["grad"].mul_(1e-20)
        before = model.values()
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        P.logra_adamw_step(P.logra_adamw_plan(model.tensors, 1), step, 1e-3)
        got = model.values()[0]
        want = before[0]["grad"] * (1e-3 / 1e-8)
        within(got["param"], before[0]["param"] - want, 3 * U * np.abs(before[0]["param"]) + 1e-3 * np.abs(want) + 1e-30, "param")


def test_what_is_not_finite_stays_in_its_elements_or_stops_its_group():
    import torch
    import paper_2405_13954_amd as P
    for bits in (32, 8):
        for norms in (False, True):
            model = Model(np.random.default_rng(8), [(3, 600, 0), (1, 50, 2)], bits)
            grad = model.dev[0]["grad"]
            grad[5], grad[600 + 7] = float("nan"), float("inf")
            before = model.values()
            out = torch.empty(3, device="cuda") if norms else None
            step = torch.zeros(1, dtype=torch.int64, device="cuda")
            P.logra_adamw_step(P.logra_adamw_plan(model.tensors, 3), step, 1e-3, norms=out)
            got = model.values()
            if norms:
                assert torch.isfinite(out).tolist() == [False, False, True] and int(step) == 1
                for k in ("param", "m", "v"):
                    assert np.array_equal(got[0][k][:2], before[0][k][:2]) and np.isfinite(got[0][k]).all()
                assert not np.array_equal(got[0]["param"][2], before[0]["param"][2])
                continue
            for k in ("param", "m", "v"):
                bad = np.argwhere(~np.isfinite(got[0][k])).tolist()
                assert bad == [[0, 5], [1, 7]], (bits, k, bad)
                assert np.isfinite(got[1][k]).all()
            assert np.isnan(got[0]["v"][0, 5]) and np.isinf(got[0]["v"][1, 7]) and np.isnan(got[0]["param"][1, 7])
            # the others of the blocks are what they would have been
            want, _ = O.adamw_step([{**x, "grad": np.where(np.isfinite(x["grad"]), x["grad"], 0.0)} for x in before], 3, 0, 1e-3)
            keep = np.isfinite(got[0]["param"])
            if bits == 8:
                assert np.array_equal(got[0]["m"][keep], want[0]["m"][keep]) and np.array_equal(got[0]["v"][keep], want[0]["v"][keep])


def test_eight_bit_blocks_of_every_size_of_value():
    # every power of two that fp32 gradients reach, and blocks at the edge of the types' largest value
    import torch
    import paper_2405_13954_amd as P
    g = np.random.default_rng(9)
    n = 256 * 70
    model = Model(g, [(1, n, 0)], 8, zero_state=True)
    grad = np.repeat(2.0 ** np.linspace(-149, 126, 70).round(), 256) * np.tile(np.where(np.arange(256) == 3, 1.75 / 0.9, g.uniform(0, 1, 256)), 70)
    model.dev[0]["grad"].copy_(torch.from_numpy(grad).float())
    before = model.values()
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    P.logra_adamw_step(P.logra_adamw_plan(model.tensors, 1), step, 1e-3, beta1=0.1, beta2=0.5, seed=12)
    got, (want,) = model.values()[0], O.adamw_step(before, 1, 0, 1e-3, 0.1, 0.5, seed=12)[0]
    for k in ("m", "v"):
        assert np.array_equal(got[k], want[k], equal_nan=True) and np.array_equal(got[k + "_scale"], want[k + "_scale"])
    assert (got["v"][0] > 0).sum() == (want["v"] > 0).sum() > n // 2


def test_rounding_is_unbiased_over_steps():
    # with the gradient at its mean value m and v stay near it, though a step adds less than the types hold: after 400
    # steps from there, the mean over 4,096 elements is within 5 of its standard deviations (each step's rounding has a
    # variance of at most a quarter of the square of the distance to the next value, an eighth, and is forgotten at 1 - beta)
    import torch
    import paper_2405_13954_amd as P
    n, value = 4096, 1.0 / 3
    mk = lambda x, t: torch.full((n,), x).to(t).cuda()  # noqa: E731
    param, grad = torch.zeros(n, device="cuda"), mk(value, torch.float32)
    m, v = mk(value * 256, torch.float8_e4m3fn), mk(value ** 2 * 65536, torch.float8_e5m2)
    ms, vs = torch.full((16,), 2.0 ** -8, device="cuda"), torch.full((16,), 2.0 ** -16, device="cuda")
    plan = P.logra_adamw_plan([P.AdamwTensor(param, grad, m, v, ms, vs)], 1)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    for _ in range(400):
        P.logra_adamw_step(plan, step, 0.0, beta1=0.9, beta2=0.99, seed=77)
    for x, s, beta, want, gap in ((m, ms, 0.9, value, 1 / 8), (v, vs, 0.99, value ** 2, 1 / 4)):
        got = float((x.double().view(16, 256) * s.double()[:, None]).mean())
        sd = want * gap / 2 / np.sqrt(1 - beta ** 2) / np.sqrt(n)
        assert abs(got - want) <= 5 * sd, (got, want, sd)


def test_reruns_streams_graphs_and_one_seed():
    import torch
    import paper_2405_13954_amd as P
    for bits in (32, 8):
        make = lambda: Model(np.random.default_rng(10), [(3, 5000, 0), (1, 777, 2)], bits)  # noqa: E731
        runs = []
        for kind in ("eager", "stream", "graph", "other seed"):
            model = make()
            step, scale = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.ones(3, device="cuda")
            plan = P.logra_adamw_plan(model.tensors, 3)
            norms = torch.empty(3, device="cuda")
            call = lambda seed=5: P.logra_adamw_step(plan, step, 1e-2, max_norm=1.0, lr_scale=scale, norms=norms, seed=seed)  # noqa: E731
            if kind == "graph":
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    call()
            side = torch.cuda.Stream()
            for k in range(4):
                scale.mul_(0.9)
                model.dev[0]["grad"].mul_(-0.5)
                torch.cuda.synchronize()
                if kind == "graph":
                    graph.replay()
                elif kind == "stream":
                    with torch.cuda.stream(side):
                        call()
                else:
                    call(6 if kind == "other seed" else 5)
                torch.cuda.synchronize()
            assert int(step) == 4
            runs.append([t.clone().view(torch.uint8) for d in model.dev for t in d.values()] + [norms.view(torch.uint8)])
        for other in runs[1:3]:
            assert all(torch.equal(a, b) for a, b in zip(runs[0], other))
        assert all(torch.equal(a, b) for a, b in zip(runs[0], runs[3])) == (bits == 32)


def test_memory_that_is_no_plan():
    import torch
    import paper_2405_13954_amd as P
    model = Model(np.random.default_rng(11), [(2, 5000, 0)], 32)
    plan = P.logra_adamw_plan(model.tensors, 2)
    before = model.values()
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    for bad in (torch.zeros_like(plan.memory), torch.full_like(plan.memory, 255)):
        P.logra_adamw_step(plan._replace(memory=bad), step, 1e-3, max_norm=1.0)
    P.logra_adamw_step(plan._replace(n_groups=1), step, 1e-3)                      # made for two groups
    P.logra_adamw_step(plan._replace(memory=plan.memory[:-256]), step, 1e-3)       # a part of it
    assert int(step) == 0 and all(np.array_equal(model.values()[0][k], before[0][k]) for k in ("param", "m", "v"))
    P.logra_adamw_step(plan, step, 1e-3)
    assert int(step) == 1


def test_plans_without_elements():
    import torch
    import paper_2405_13954_amd as P
    empty = torch.empty(0, device="cuda")
    step, norms = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((2,), 5.0, device="cuda")
    for tensors in ([], [P.AdamwTensor(empty, empty, empty, empty)]):
        P.logra_adamw_step(P.logra_adamw_plan(tensors, 2), step, 1e-3, norms=norms)
        assert norms.tolist() == [0.0, 0.0]
    assert int(step) == 2


def test_refusals():
    import torch
    import paper_2405_13954_amd as P
    x = lambda n=8: torch.zeros(n, device="cuda")  # noqa: E731
    p, g, m, v = x(), x(), x(), x()
    ok = P.AdamwTensor(p, g, m, v)
    for bad in (ok._replace(grad=p), ok._replace(v=m), ok._replace(m=g), ok._replace(slices=3), ok._replace(m_scale=x(1)),
                ok._replace(first_group=1), ok._replace(first_group=-1), ok._replace(grad=x(9)), ok._replace(work=x()),
                ok._replace(grad=x().cpu()), ok._replace(param=x(16)[::2])):
        with pytest.raises((P.LograError, ValueError)):
            P.logra_adamw_plan([bad], 1)
    with pytest.raises(P.LograError):
        P.logra_adamw_plan([ok, P.AdamwTensor(p, g, x(), x())], 1)      # the same parameter twice
    with pytest.raises(P.LograError):
        big = x(16)
        P.logra_adamw_plan([P.AdamwTensor(big[:8], g, m, v), P.AdamwTensor(big[7:15], g, x(), x())], 1)
    P.logra_adamw_plan([ok, P.AdamwTensor(x(), g, x(), x())], 1)        # one gradient of two parameters
    plan, step = P.logra_adamw_plan([ok], 1), torch.zeros(1, dtype=torch.int64, device="cuda")
    for kw in (dict(beta1=1.0), dict(beta2=1.0), dict(beta1=-0.1), dict(eps=0.0), dict(eps=float("nan")), dict(weight_decay=-1.0),
               dict(max_norm=-1.0), dict(max_norm=float("nan"))):
        with pytest.raises(P.LograError):
            P.logra_adamw_step(plan, step, 1e-3, **kw)
    with pytest.raises(P.LograError):
        P.logra_adamw_step(plan, step, float("inf"))
    with pytest.raises(P.LograError):
        P.logra_adamw_step(plan, step.cpu(), 1e-3)
    with pytest.raises(ValueError):
        P.logra_adamw_step(plan, step.int(), 1e-3)
    with pytest.raises(ValueError):
        P.logra_adamw_step(plan, step, 1e-3, lr_scale=x(2))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    memory = torch.empty_like(plan.memory)
    with torch.cuda.graph(graph):
        with pytest.raises(P.LograError, match="captur"):
            P.logra_adamw_plan([ok], 1)
        memory.zero_()
