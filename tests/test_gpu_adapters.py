"""Adapters of many requests (logra_adapter_*) against the float64 oracle.

Tolerances are bounds, derived before any run.  With eps = 2^-23 (one fp32 step; matrix-core sums may truncate) and
|.| the sum of the absolute values of a result's terms, as the oracle returns it:
  u       n_in + 8 additions                                  (n_in + 8) eps |u|
  dA, dB  the sums over rows and the long axis, and the
          products' roundings (u and du keep 24 bits)         (rows + n + 16) eps |dW|
  y, dx   the sums, u's 16 significant bits as an operand
          (2^-16 |y|), and one rounding to the output type    ((n + rank + 8) eps + 2^-16) |y| + ulp/2 |y*|
where ulp/2 is 2^-8 of the value for bf16 and 2^-24 for fp32, and the 2^-16 is absent in fp32.
"""
import numpy as np
import pytest

from oracle import adapters as O

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -23
SENTINEL = 12345.0


def _dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _mk(g, shape, std, dtype, pad=0, fill=None):
    """(device view of shape, float64 copy) of rounded normal values; rows carry `pad` further sentinel columns."""
    import torch
    t = torch.from_numpy(g.standard_normal(shape).astype(np.float32) * np.float32(std)).to(_dt(dtype))
    full = torch.full((*shape[:-1], shape[-1] + pad), SENTINEL, dtype=_dt(dtype))
    full[..., :shape[-1]] = t
    full = full.cuda()
    return full[..., :shape[-1]], t.double().numpy(), full


def _ids(g, rows, n, kind):
    if kind == "none":
        return np.full(rows, -1, dtype=np.int32)
    if kind == "one":
        return np.full(rows, n - 1, dtype=np.int32)
    if kind == "mixed":      # any order, with values on both sides of the range
        return g.integers(-1, n + 1, rows).astype(np.int32)
    ids = np.sort(g.integers(0, n, rows)).astype(np.int32)       # requests, with padding at the end of each
    ids[g.random(rows) < 0.2] = -1
    return ids


def _case(seed, rows, n_in, n_out, rank, n, dtype, ids="mixed", p=0.0, base=True, scale=True, pad=0):
    import torch
    g = np.random.default_rng([seed, rows, n_in, n_out, rank, n])
    c = {"n": n, "rank": rank, "dtype": dtype, "p": p, "seed": 0xABCDEF0123456789, "offset": 3 << 32 | 5}
    c["ids"] = _ids(g, rows, n, ids)
    c["x"], c["x64"], _ = _mk(g, (rows, n_in), 1.0, dtype, pad)
    c["dy"], c["dy64"], _ = _mk(g, (rows, n_out), 0.1, dtype, pad)
    c["a"], c["a64"], _ = _mk(g, (n, rank, n_in), n_in ** -0.5, dtype)
    c["b"], c["b64"], _ = _mk(g, (n, rank, n_out), rank ** -0.5, dtype)
    c["base"], c["base64"], c["basefull"] = _mk(g, (rows, n_out), 1.0, dtype, pad) if base else (None, None, None)
    c["back"], c["back64"], c["backfull"] = _mk(g, (rows, n_in), 0.1, dtype, pad) if base else (None, None, None)
    c["scale64"] = g.uniform(0.25, 2.0, n).astype(np.float32) if scale else None
    c["scale"] = torch.from_numpy(c["scale64"]).cuda() if scale else None
    c["f"] = O.drop_factor(rows, n_in, p, c["seed"], c["offset"]) if p else None
    return c


def _plan(c):
    import torch
    import paper_2405_13954_amd as P
    return P.logra_adapter_plan(torch.from_numpy(c["ids"]).cuda(), c["n"])


def _out(rows, cols, dtype, pad):
    import torch
    full = torch.full((rows, cols + pad), SENTINEL, dtype=dtype, device="cuda")
    return full[:, :cols], full


def _half_ulp(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24


def _near(got, want, bound, what):
    got = got.detach().double().cpu().numpy()
    worst = np.max(np.abs(got - want) - bound) if want.size else 0.0
    assert np.all(np.isfinite(got)) and worst <= 0.0, f"{what}: {worst:.3e} beyond the bound"


def _y_bound(c, y, ya, n):
    return ((n + c["rank"] + 8) * EPS + (2.0 ** -16 if c["dtype"] == "bf16" else 0.0)) * ya + _half_ulp(c["dtype"]) * np.abs(y)


def _forward(c, plan, inplace=False, pad=0, want_u=True, **kw):
    import torch
    import paper_2405_13954_amd as P
    rows, n_out = c["x"].shape[0], c["b"].shape[2]
    if inplace:
        y, full = c["base"], c["basefull"]
    else:
        y, full = _out(rows, n_out, _dt(c["dtype"]), pad)
    u = torch.full((rows, c["rank"]), SENTINEL, device="cuda") if want_u else None
    P.logra_adapter_forward(c["x"], c["a"], c["b"], plan, y, base=c["base"], scale=c["scale"], u=u, p=c["p"],
                            seed=c["seed"], offset=c["offset"], **kw)
    return y, u, full


def _check_forward(c, pad=0, inplace=False):
    print("[adapter fwd]", {k: c[k] for k in ("n", "rank", "dtype", "p")}, tuple(c["x"].shape), tuple(c["b"].shape), flush=True)
    want, u64, ya, ua = O.adapter_forward(c["x64"], c["a64"], c["b64"], c["ids"], c["base64"], c["scale64"], c["f"])
    y, u, full = _forward(c, _plan(c), inplace, pad)
    n_in = c["x"].shape[1]
    _near(u, u64, (n_in + 8) * EPS * ua, "u")
    _near(y, want, _y_bound(c, want, ya, n_in), "y")
    if pad:
        assert bool((full[:, y.shape[1]:] == SENTINEL).all()), "store between the rows of y"
    none = (c["ids"] < 0) | (c["ids"] >= c["n"])
    if c["base"] is not None:
        assert np.array_equal(y.double().cpu().numpy()[none], c["base64"][none])
    return y, u


SHAPES = [   # rows, n_in, n_out, rank, adapters
    (1, 8, 8, 1, 1), (1, 264, 40, 16, 3), (2, 64, 1032, 9, 5), (17, 72, 248, 33, 4), (33, 512, 64, 64, 2),
    (70, 1000, 136, 100, 3), (257, 136, 264, 16, 1), (300, 264, 520, 128, 2), (515, 776, 88, 17, 40), (64, 4096, 8, 8, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype):
    _check_forward(_case(1, *shape, dtype), pad=8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ids", ["none", "one", "requests"])
def test_forward_groups(ids, dtype):
    _check_forward(_case(2, 130, 136, 200, 16, 6, dtype, ids=ids, pad=16), pad=0)
    _check_forward(_case(2, 130, 136, 200, 16, 6, dtype, ids=ids, base=False, scale=False), pad=0)
    _check_forward(_case(2, 130, 136, 200, 16, 6, dtype, ids=ids, pad=8), inplace=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(5, 72, 40, 4, 2), (150, 520, 64, 16, 3), (90, 264, 64, 64, 2), (40, 200, 64, 128, 1)])
def test_forward_dropout(shape, dtype):
    _check_forward(_case(3, *shape, dtype, p=0.2))


def _check_backward(c, accumulate=False, inplace=False, want_dx=True, pad=0):
    import torch
    import paper_2405_13954_amd as P
    print("[adapter bwd]", {k: c[k] for k in ("n", "rank", "dtype", "p")}, tuple(c["x"].shape), tuple(c["b"].shape), flush=True)
    rows, n_in, n_out, n, rank = *c["x"].shape, c["b"].shape[2], c["n"], c["rank"]
    g = np.random.default_rng(7)
    u64 = g.standard_normal((rows, rank)).astype(np.float32)
    (da, db, dx), (daa, dba, dxa) = O.adapter_backward(c["x64"], c["dy64"], c["a64"], c["b64"], c["ids"],
                                                        u64.astype(np.float64), c["back64"], c["scale64"], c["f"])
    start = [g.standard_normal(s).astype(np.float32) for s in (da.shape, db.shape)]
    gda, gdb = (torch.from_numpy(s).cuda() for s in start)
    gdx, full = (c["back"], c["backfull"]) if inplace else _out(rows, n_in, _dt(c["dtype"]), pad)
    P.logra_adapter_backward(c["x"], c["dy"], c["a"], c["b"], _plan(c), torch.from_numpy(u64).cuda(), gda, gdb,
                             dx=gdx if want_dx else None, base=c["back"] if want_dx else None, scale=c["scale"],
                             p=c["p"], seed=c["seed"], offset=c["offset"], accumulate=accumulate)
    if accumulate:
        da, db, daa, dba = da + start[0], db + start[1], daa + np.abs(start[0]), dba + np.abs(start[1])
    _near(gda, da, (rows + n_out + 16) * EPS * daa, "dA")
    _near(gdb, db, (rows + n_in + 16) * EPS * dba, "dB")
    if want_dx:
        _near(gdx, dx, _y_bound(c, dx, dxa, n_out), "dx")
        if pad:
            assert bool((full[:, n_in:] == SENTINEL).all()), "store between the rows of dx"
    return gda, gdb, gdx


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, dtype):
    _check_backward(_case(4, *shape, dtype), pad=8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ids", ["none", "one", "requests"])
def test_backward_groups(ids, dtype):
    shape = (330, 136, 200, 16, 6)
    _check_backward(_case(5, *shape, dtype, ids=ids, pad=16), accumulate=True)
    _check_backward(_case(5, *shape, dtype, ids=ids, base=False, scale=False), want_dx=ids != "one")
    _check_backward(_case(5, *shape, dtype, ids=ids, pad=8), inplace=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(5, 72, 40, 4, 2), (150, 520, 64, 16, 3), (90, 264, 64, 64, 2), (40, 200, 64, 128, 1)])
def test_backward_dropout(shape, dtype):
    _check_backward(_case(6, *shape, dtype, p=0.2))


def test_gradients_against_differences_of_the_kernels():
    # fp32: y is linear in a, b and x, so a central difference of the forward kernel is the gradient to the rounding
    # of the forward pass; the bound is that of y's errors in sum(y * dy), twice, and of the gradient's in sum(grad * e)
    import torch
    import paper_2405_13954_amd as P
    c = _case(8, 60, 64, 48, 8, 3, "f32", p=0.1)
    plan, (rows, n_in) = _plan(c), c["x"].shape
    _, u, _ = _forward(c, plan)
    grads = [torch.empty(3, 8, 64, device="cuda"), torch.empty(3, 8, 48, device="cuda"), torch.empty(rows, n_in, device="cuda")]
    P.logra_adapter_backward(c["x"], c["dy"], c["a"], c["b"], plan, u, grads[0], grads[1], dx=grads[2], scale=c["scale"],
                             p=c["p"], seed=c["seed"], offset=c["offset"])
    ids = torch.from_numpy(c["ids"]).cuda()
    live = ((ids >= 0) & (ids < 3))[:, None]
    for name, grad in zip(("a", "b", "x"), grads):
        e = torch.randn(c[name].shape, generator=torch.Generator().manual_seed(1)).cuda()
        ys, mag = [], 0.0
        for k in (0.5, -0.5):
            t = {**c, name: c[name] + k * e, "base": None}
            ys.append(_forward(t, plan)[0].double())
            ab = {q: t[q].abs() for q in ("x", "a", "b")}
            mag += float((_forward({**t, **ab}, plan)[0].double().abs() * c["dy"].double().abs()).sum())
        diff = float(((ys[0] - ys[1]) * c["dy"].double()).sum())
        dot = float((grad.double() * e.double()).where(live, torch.zeros((), device="cuda", dtype=torch.double)).sum()
                    if name == "x" else (grad.double() * e.double()).sum())
        assert abs(diff - dot) <= 4 * (64 + 48 + 60 + 32) * EPS * mag, (name, diff, dot)


def test_masked_rows_and_dropped_elements_are_never_used():
    import torch
    c = _case(9, 50, 136, 72, 12, 3, "bf16", p=0.5)
    none = torch.from_numpy((c["ids"] < 0) | (c["ids"] >= 3))
    c["x"][none.cuda()] = float("nan")
    c["x64"][none.numpy()] = 0.0
    c["dy"][none.cuda()] = float("inf")
    c["dy64"][none.numpy()] = 0.0
    gone = (c["f"] == 0.0) & ~none.numpy()[:, None]
    c["x"][torch.from_numpy(gone).cuda()] = float("nan")
    _check_forward(c)
    _check_backward(c)


def test_nan_stays_in_its_row():
    import torch
    c = _case(10, 40, 64, 64, 16, 2, "bf16", ids="one")
    c["x"][7, 3], c["x"][9, 5] = float("nan"), float("inf")
    y, u, _ = _forward(c, _plan(c))
    bad = ~torch.isfinite(y).all(1)
    assert bad.nonzero()[:, 0].tolist() == [7, 9] and torch.isnan(y[7]).all()


@pytest.mark.parametrize("rows", [1, 63, 4096, 4097, 20000])
def test_plan_groups_any_order(rows):
    # the plan's effect on many rows in any order: every row gets its own adapter (rank 1, n = 8: y is a product)
    import torch
    import paper_2405_13954_amd as P
    for n in (1, 37, 1023):
        g = torch.Generator().manual_seed(rows + n)
        ids = torch.randint(-2, n + 2, (rows,), generator=g, dtype=torch.int32).cuda()
        x = torch.randn(rows, 8, generator=g).cuda()
        a, b = torch.randn(n, 1, 8, generator=g).cuda(), torch.randn(n, 1, 8, generator=g).cuda()
        y = torch.empty(rows, 8, device="cuda")
        P.logra_adapter_forward(x, a, b, P.logra_adapter_plan(ids, n), y)
        at = ids.long().clamp(0, n - 1)
        want = (a.double()[at, 0] * x.double()).sum(1, keepdim=True) * b.double()[at, 0]
        mag = (a.double()[at, 0] * x.double()).abs().sum(1, keepdim=True) * b.double()[at, 0].abs()
        live = ((ids >= 0) & (ids < n))[:, None]
        want = torch.where(live, want, 0.0)
        assert bool(((y.double() - want).abs() <= 32 * EPS * mag).all()), (rows, n)
        assert bool((y[~live[:, 0]] == 0).all())


def test_reruns_are_bitwise_equal_and_other_plans_do_nothing():
    import torch
    import paper_2405_13954_amd as P
    c = _case(11, 700, 264, 136, 16, 5, "bf16", p=0.1)
    first = [t.clone() for t in (*_check_forward(c), *_check_backward(c))]
    again = [*_check_forward(c), *_check_backward(c)]
    assert all(torch.equal(p, q) for p, q in zip(first, again))
    # a plan for other rows, and memory that is no plan
    for plan in (P.logra_adapter_plan(torch.zeros(900, dtype=torch.int32, device="cuda"), 5),
                 torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")):
        y, u, _ = _forward(c, plan)
        assert bool((y == SENTINEL).all()) and bool((u == SENTINEL).all())


def test_no_rows():
    import torch
    import paper_2405_13954_amd as P
    x, dy = torch.empty(0, 16, device="cuda"), torch.empty(0, 24, device="cuda")
    a, b = torch.randn(2, 3, 16, device="cuda"), torch.randn(2, 3, 24, device="cuda")
    plan = P.logra_adapter_plan(torch.empty(0, dtype=torch.int32, device="cuda"), 2)
    P.logra_adapter_forward(x, a, b, plan, dy)
    da, db, u = torch.ones_like(a), torch.ones_like(b), torch.empty(0, 3, device="cuda")
    P.logra_adapter_backward(x, dy, a, b, plan, u, da, db, accumulate=True)
    assert bool((da == 1).all()) and bool((db == 1).all())
    P.logra_adapter_backward(x, dy, a, b, plan, u, da, db)
    assert bool((da == 0).all()) and bool((db == 0).all())


def test_offsets_beyond_32_bits():
    # 40 rows at a stride of 2^27 elements: byte offsets to 2^33 and 2^34, the rows next to the last among them
    import torch
    for dtype in ("bf16", "f32"):
        c = _case(12, 40, 64, 32, 16, 2, dtype)
        wide = torch.empty(40 << 27 if dtype == "bf16" else 20 << 27, dtype=_dt(dtype), device="cuda").view(40, -1)
        x, base = wide[:, 8:72], wide[:, 128:160]
        x.copy_(c["x"])
        base.copy_(c["base"])
        c["x"], c["base"] = x, base
        _check_forward(c)
        dy, back = wide[:, 256:288], wide[:, 512:576]
        dy.copy_(c["dy"])
        back.copy_(c["back"])
        c["dy"], c["back"] = dy, back
        _check_backward(c)
        del wide, x, base, dy, back, c


def test_other_stream_and_graph():
    import torch
    import paper_2405_13954_amd as P
    c = _case(13, 200, 264, 136, 16, 3, "bf16", p=0.1)
    plan = _plan(c)
    want = [t.clone() for t in _forward(c, plan)[:2]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _forward(c, _plan(c))[:2]
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    ids = torch.from_numpy(c["ids"]).cuda()
    y, u = torch.empty_like(want[0]), torch.empty_like(want[1])
    da, db, dx = torch.empty(3, 16, 264, device="cuda"), torch.empty(3, 16, 136, device="cuda"), torch.empty_like(c["back"])
    ws = torch.empty(P.logra_adapter_ws_size(200, 264, 136, 16, 3), dtype=torch.uint8, device="cuda")
    kw = dict(scale=c["scale"], p=c["p"], seed=c["seed"], offset=c["offset"], ws=ws)

    def step():
        P.logra_adapter_plan(ids, 3, plan=plan)
        P.logra_adapter_forward(c["x"], c["a"], c["b"], plan, y, base=c["base"], u=u, **kw)
        P.logra_adapter_backward(c["x"], c["dy"], c["a"], c["b"], plan, u, da, db, dx=dx, base=c["back"], **kw)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        ids.copy_(torch.roll(torch.from_numpy(c["ids"]), k))     # other rows for every replay
        c["x"].mul_(1.25)
        step()
        want = [t.clone() for t in (y, u, da, db, dx)]
        for t in (y, u, da, db, dx):
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((y, u, da, db, dx), want)), f"replay {k}"


def test_binding_refuses():
    import torch
    import paper_2405_13954_amd as P
    c = _case(14, 10, 64, 32, 4, 2, "bf16")
    plan = _plan(c)
    bad = [dict(x=c["x"].float()), dict(a=c["a"][:, :, :32]), dict(b=c["b"].float()), dict(base=c["base"][:5]),
           dict(scale=torch.ones(3, device="cuda")), dict(x=c["x"].t()[:10])]
    for change in bad:
        with pytest.raises(ValueError):
            _forward({**c, **change}, plan)
    for change, status in ((dict(p=1.0), P.ERR_INVALID_ARG), (dict(p=-0.1), P.ERR_INVALID_ARG)):
        with pytest.raises(P.LograError) as e:
            _forward({**c, **change}, plan)
        assert e.value.status == status
    with pytest.raises(P.LograError) as e:
        _forward(c, plan[:256])
    assert e.value.status == P.ERR_WORKSPACE
    with pytest.raises(P.LograError) as e:
        _forward(c, plan, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == P.ERR_WORKSPACE
    with pytest.raises(P.LograError) as e:
        _forward({**c, "x": torch.empty(10, 64, dtype=torch.bfloat16)}, plan)     # host memory
    assert e.value.status == P.ERR_INVALID_ARG
    with pytest.raises(TypeError):
        P.logra_adapter_plan(torch.zeros(4, dtype=torch.int64, device="cuda"), 2)
