"""The operators that train and serve adapters beside a frozen model, as they are timed and compared.

A data-valuation program ends in a choice of training data, and the choice is tried out: adapters are trained on
the chosen subsets, many of them at once beside the one frozen model, and the responses of each are compared.  The
cases are the calls that such a program makes for one linear layer or for the last layer's logits:

  adapter_forward   y = base + s_a B_a^T A_a drop(x) for rows of many requests, each with its own adapter a
  adapter_backward  the gradients of that: dA, dB of every adapter and dx = base + (what the adapter sends back)
  dropout           residual + drop(x), the mask drawn from a counter and never stored
  token_loss        cross-entropy of each token's logits and its gradient

`run` computes them in elementary torch operations, in 32 bits, or (with `own`) by the library's entry points.
`exact` computes them in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One new token each of 8 requests, 8 adapters of rank 16, at a 4096 -> 4096 projection: the smallest
        # serving step, where launches count and not bytes.
        {"name": "serve_8", "kind": "adapter_forward", "rows": 8, "requests": 8, "adapters": 8, "n_in": 4096,
         "n_out": 4096, "rank": 16, "dtype": "bf16", "p": 0.0, "train": False, "none": False, "pad": 0},
        # One new token each of 96 requests that share 64 adapters, some with none, at the wide projection of a
        # block: the adapters' weights are most of the bytes.
        {"name": "serve_96_wide", "kind": "adapter_forward", "rows": 96, "requests": 96, "adapters": 64, "n_in": 4096,
         "n_out": 14336, "rank": 16, "dtype": "bf16", "p": 0.0, "train": False, "none": True, "pad": 0},
        # Prompts of 5 requests, 1,999 rows in all, rank 64 at a narrow projection, rows in a wider buffer.
        {"name": "prompt_r64", "kind": "adapter_forward", "rows": 1999, "requests": 5, "adapters": 5, "n_in": 4096,
         "n_out": 1024, "rank": 64, "dtype": "bf16", "p": 0.0, "train": False, "none": True, "pad": 64},
        # A training step's forward pass: 16 sequences of 1,024 tokens for 8 subsets' adapters, dropout on their input.
        {"name": "train_fwd", "kind": "adapter_forward", "rows": 16384, "requests": 16, "adapters": 8, "n_in": 4096,
         "n_out": 4096, "rank": 16, "dtype": "bf16", "p": 0.05, "train": True, "none": False, "pad": 0},
        # A small fp32 model: 509 rows of 3 adapters of odd rank.
        {"name": "train_fwd_f32", "kind": "adapter_forward", "rows": 509, "requests": 7, "adapters": 3, "n_in": 768,
         "n_out": 2304, "rank": 9, "dtype": "f32", "p": 0.1, "train": True, "none": True, "pad": 4},
        # The backward pass of the training step above, padding rows among the sequences.
        {"name": "train_bwd", "kind": "adapter_backward", "rows": 16384, "requests": 16, "adapters": 8, "n_in": 4096,
         "n_out": 4096, "rank": 16, "dtype": "bf16", "p": 0.05, "none": True, "pad": 0},
        # The backward pass of a short ragged batch at rank 64 into a narrow layer's input.
        {"name": "train_bwd_r64", "kind": "adapter_backward", "rows": 2047, "requests": 9, "adapters": 4, "n_in": 4096,
         "n_out": 1024, "rank": 64, "dtype": "bf16", "p": 0.0, "none": True, "pad": 0},
        # The backward pass of the small fp32 model.
        {"name": "train_bwd_f32", "kind": "adapter_backward", "rows": 509, "requests": 7, "adapters": 3, "n_in": 768,
         "n_out": 2304, "rank": 9, "dtype": "f32", "p": 0.1, "none": True, "pad": 4},
        # Dropout of a block's output before it joins the residual stream.
        {"name": "dropout_residual", "kind": "dropout", "rows": 16384, "cols": 4096, "dtype": "bf16", "p": 0.1,
         "residual": True, "pad": 0},
        # Dropout alone on a small fp32 tensor of odd width (the backward pass is the same call on the gradient).
        {"name": "dropout_f32_odd", "kind": "dropout", "rows": 333, "cols": 1001, "dtype": "f32", "p": 0.25,
         "residual": False, "pad": 3},
        # Losses and logit gradients of a batch at a large vocabulary, a part of the tokens masked.
        {"name": "loss_128k", "kind": "token_loss", "rows": 2048, "vocab": 128000, "dtype": "bf16", "masked": 0.2,
         "weighted": True, "pad": 0},
        # A short sequence at an odd vocabulary in fp32.
        {"name": "loss_f32_odd", "kind": "token_loss", "rows": 61, "vocab": 50001, "dtype": "f32", "masked": 0.0,
         "weighted": False, "pad": 3},
    ]


def _logint(rng, lo, hi, mult=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(mult, v // mult * mult)


def draw(rng):
    kind = rng.choice(("adapter_forward", "adapter_forward", "adapter_backward", "adapter_backward", "dropout",
                       "token_loss"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind == "dropout":
        cols = _logint(rng, 33, 16384)
        return {"kind": kind, "rows": min(_logint(rng, 1, 16384), 60_000_000 // cols), "cols": cols, "dtype": dtype,
                "p": rng.choice((0.0, 0.05, 0.1, 0.5)), "residual": rng.random() < 0.5,
                "pad": -cols % 8 + 8 * rng.randint(0, 2)}
    if kind == "token_loss":
        vocab = _logint(rng, 500, 200_000)
        return {"kind": kind, "rows": max(1, min(_logint(rng, 1, 4096), 120_000_000 // vocab)), "vocab": vocab,
                "dtype": dtype, "masked": rng.choice((0.0, 0.2, 0.7)), "weighted": rng.random() < 0.5,
                "pad": -vocab % 8}
    rows = _logint(rng, 1, 16384)
    most = 60_000_000 // rows
    n_in = min(_logint(rng, 64, 14336, 8), max(64, most // 8 * 8))
    n_out = min(_logint(rng, 64, 14336, 8), max(64, (most - n_in) // 8 * 8))
    adapters = _logint(rng, 1, 64)
    case = {"kind": kind, "rows": rows, "requests": min(rows, _logint(rng, 1, 128)), "adapters": adapters,
            "n_in": n_in, "n_out": n_out, "rank": rng.choice((1, 4, 8, 9, 16, 16, 32, 48, 64)), "dtype": dtype,
            "p": rng.choice((0.0, 0.0, 0.05, 0.1))}
    if kind == "adapter_forward":
        case["train"] = rng.random() < 0.5
        if not case["train"]:
            case["p"] = 0.0
    return {**case, "none": rng.random() < 0.5, "pad": rng.choice((0, 0, 8, 64))}


# -------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(np.random.SeedSequence([int(seed), 977]).generate_state(1)[0]))
    return g


def _rand(g, rows, cols, std, dtype, pad=0):
    """[rows, cols] of N(0, std^2), as a view of rows with `pad` further columns."""
    t = torch.empty(rows, cols + pad, dtype=dtype, device=DEV)
    for at in range(0, rows, 4096):
        part = t[at:at + 4096]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV) * std)
    return t[:, :cols]


def _row_adapters(case, seed):
    """The adapter of each row: contiguous requests of ragged lengths; -1 for a request that has none and for
    padding rows at the end of some requests."""
    r = np.random.default_rng([int(seed), 31])
    rows, n = case["rows"], case["requests"]
    cuts = np.sort(r.choice(np.arange(1, rows), n - 1, replace=False)) if n > 1 else np.array([], dtype=np.int64)
    of_request = r.permutation(np.arange(n) % case["adapters"])
    ids = np.empty(rows, dtype=np.int32)
    for a, lo, hi in zip(of_request, [0, *cuts], [*cuts, rows]):
        ids[lo:hi] = a
        if case["none"]:
            if n > 4 and r.random() < 0.15:
                ids[lo:hi] = -1
            elif hi - lo > 4 and r.random() < 0.5:
                ids[hi - int(r.integers(1, (hi - lo) // 2)):hi] = -1
    return torch.from_numpy(ids)


def prepare(case, seed):
    g, dtype = _gen(seed), DTYPES[case["dtype"]]
    s = dict(case)
    rows, pad = case["rows"], case["pad"]
    s["seed"], s["offset"] = 0x9E3779B97F4A7C15 ^ int(seed), (int(seed) % 1000) << 33 | 7
    if case["kind"] == "dropout":
        s["x"] = _rand(g, rows, case["cols"], 1.0, dtype, pad)
        s["residual"] = _rand(g, rows, case["cols"], 2.0, dtype, pad) if case["residual"] else None
        s["out"] = torch.empty(rows, case["cols"] + pad, dtype=dtype, device=DEV)[:, :case["cols"]]
        return s
    if case["kind"] == "token_loss":
        # logits of a trained model: a wide spread, and the target among the likelier tokens
        s["logits"] = _rand(g, rows, case["vocab"], 2.5, dtype, pad)
        target = torch.randint(case["vocab"], (rows,), generator=g, device=DEV)
        off = torch.rand(rows, generator=g, device=DEV) < case["masked"]
        s["target"] = torch.where(off, -1, target)
        s["weight"] = torch.rand(rows, generator=g, device=DEV) + 0.5 if case["weighted"] else None
        s["loss"] = torch.empty(rows, dtype=torch.float32, device=DEV)
        s["dlogits"] = torch.empty(rows, case["vocab"] + pad, dtype=dtype, device=DEV)[:, :case["vocab"]]
        return s
    n_in, n_out, rank, n = case["n_in"], case["n_out"], case["rank"], case["adapters"]
    s["ids"] = _row_adapters(case, seed).to(DEV)
    s["x"] = _rand(g, rows, n_in, 1.0, dtype, pad)
    s["a"] = _rand(g, n * rank, n_in, n_in ** -0.5, dtype).view(n, rank, n_in)
    s["b"] = _rand(g, n * rank, n_out, 0.5 * rank ** -0.5, dtype).view(n, rank, n_out)
    s["scale"] = torch.rand(n, generator=g, device=DEV) * 1.5 + 0.5
    empty32 = lambda *shape: torch.empty(shape, dtype=torch.float32, device=DEV)  # noqa: E731
    if case["kind"] == "adapter_forward":
        s["base"] = _rand(g, rows, n_out, 1.0, dtype, pad)
        s["y"] = torch.empty(rows, n_out, dtype=dtype, device=DEV)
        s["u"] = empty32(rows, rank) if case["train"] else None
    else:
        s["dy"] = _rand(g, rows, n_out, 1e-2, dtype, pad)
        s["base"] = _rand(g, rows, n_in, 1e-2, dtype, pad)
        s["dx"] = torch.empty(rows, n_in, dtype=dtype, device=DEV)
        # A_a drop(x), as the forward pass left it
        s["u"] = _rand(g, rows, rank, 1.0, torch.float32).masked_fill(s["ids"][:, None] < 0, 0.0)
        s["da"], s["db"] = empty32(n, rank, n_in), empty32(n, rank, n_out)
    if own:
        # the grouping of the rows by adapter, made once for a batch and used by all its layers, and the
        # workspace that these share
        import paper_2405_13954_amd as P
        s["plan"] = P.logra_adapter_plan(s["ids"], n)
        s["ws"] = torch.empty(max(1, P.logra_adapter_ws_size(rows, n_in, n_out, rank, n)), dtype=torch.uint8,
                              device=DEV)
    return s


# ------------------------------------------------------------- the plain form
def _mulhilo(a, b):
    """High and low words of the 64-bit product of 32-bit words held in int64."""
    p = a * b
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _keep(rows, cols, p, seed, offset):
    """Which elements of a rows x cols matrix stay: Philox4x32-7 (Salmon et al. 2011) of the counter
    (column / 8, row, offset), 16 bits for each of the 8 columns."""
    c = torch.arange((cols + 7) // 8, device=DEV)[None, :].expand(rows, -1)
    r = torch.arange(rows, device=DEV)[:, None].expand_as(c)
    w = [c, r, torch.full_like(c, offset & 0xFFFFFFFF), torch.full_like(c, offset >> 32 & 0xFFFFFFFF)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF
    for _ in range(7):
        h0, l0 = _mulhilo(w[0], 0xD2511F53)
        h1, l1 = _mulhilo(w[2], 0xCD9E8D57)
        w = [h1 ^ w[1] ^ k0, l1, h0 ^ w[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    bits = torch.stack([w[0] & 0xFFFF, w[0] >> 16, w[1] & 0xFFFF, w[1] >> 16, w[2] & 0xFFFF, w[2] >> 16,
                        w[3] & 0xFFFF, w[3] >> 16], dim=-1).view(rows, -1)[:, :cols]
    return bits >= round(p * 65536)


def _drop(x, s):
    """drop(x): kept elements times 1 / (1 - p), zeros elsewhere."""
    if s["p"] == 0.0:
        return x
    kept = _keep(x.shape[0], x.shape[1], s["p"], s["seed"], s["offset"])
    return torch.where(kept, x * (65536 / (65536 - round(s["p"] * 65536))), 0.0)


def _plain_adapter(s):
    n, rank = s["adapters"], s["rank"]
    x, a, b = s["x"].float(), s["a"].float().view(n * rank, -1), s["b"].float().view(n * rank, -1)
    mine = s["ids"][:, None, None] == torch.arange(n, device=DEV)[None, :, None]
    scale = s["scale"][None, :, None]
    if s["kind"] == "adapter_forward":
        u = torch.where(mine, (_drop(x, s) @ a.T).view(-1, n, rank), 0.0)
        y = (s["base"].float() + (u * scale).view(-1, n * rank) @ b).to(s["base"].dtype)
        return {"y": y, "u": u.sum(1)} if s["train"] else {"y": y}
    dy = s["dy"].float()
    du = torch.where(mine, (dy @ b.T).view(-1, n, rank) * scale, 0.0).view(-1, n * rank)
    u = torch.where(mine, s["u"][:, None, :] * scale, 0.0).view(-1, n * rank)
    return {"da": (du.T @ _drop(x, s)).view(n, rank, -1), "db": (u.T @ dy).view(n, rank, -1),
            "dx": (s["base"].float() + _drop(du @ a, s)).to(s["base"].dtype)}


def _plain_loss(s):
    z, target = s["logits"].float(), s["target"]
    live = target >= 0
    at = target.clamp(min=0)[:, None]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    weight = live.float() if s["weight"] is None else torch.where(live, s["weight"], 0.0)
    loss = torch.where(live, weight * (torch.log(total) + top - z.gather(1, at))[:, 0], 0.0)
    grad = e / total
    grad.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
    grad = torch.where(live[:, None], grad * weight[:, None], 0.0)
    return {"loss": loss, "dlogits": grad.to(s["logits"].dtype)}


# ------------------------------------------------------------- the library
def _own(s):
    import paper_2405_13954_amd as P
    if s["kind"] == "adapter_forward":
        P.logra_adapter_forward(s["x"], s["a"], s["b"], s["plan"], s["y"], base=s["base"], scale=s["scale"],
                                u=s["u"], p=s["p"], seed=s["seed"], offset=s["offset"], ws=s["ws"])
        return {"y": s["y"], "u": s["u"]} if s["train"] else {"y": s["y"]}
    if s["kind"] == "adapter_backward":
        P.logra_adapter_backward(s["x"], s["dy"], s["a"], s["b"], s["plan"], s["u"], s["da"], s["db"], dx=s["dx"],
                                 base=s["base"], scale=s["scale"], p=s["p"], seed=s["seed"], offset=s["offset"],
                                 ws=s["ws"])
        return {"da": s["da"], "db": s["db"], "dx": s["dx"]}
    if s["kind"] == "dropout":
        P.logra_dropout(s["x"], s["out"], s["p"], s["seed"], s["offset"], residual=s["residual"])
        return {"out": s["out"]}
    P.logra_token_loss(s["logits"], s["target"], s["loss"], dlogits=s["dlogits"], weight=s["weight"])
    return {"loss": s["loss"], "dlogits": s["dlogits"]}


def run(s):
    if own:
        return _own(s)
    if s["kind"] == "dropout":
        out = _drop(s["x"].float(), s)
        out = out if s["residual"] is None else s["residual"].float() + out
        return {"out": out.to(s["x"].dtype)}
    if s["kind"] == "token_loss":
        return _plain_loss(s)
    return _plain_adapter(s)


# -------------------------------------------------------------------- floors
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    rows = case["rows"]
    if case["kind"] == "dropout":
        n = rows * case["cols"]
        return {"bytes": n * es * (3 if case["residual"] else 2), "flops": 2 * n}
    if case["kind"] == "token_loss":
        n = rows * case["vocab"]  # the rows that are masked are written, and not read
        return {"bytes": n * es * (2 - case["masked"]) + rows * 16, "flops": 4 * n}
    n_in, n_out, rank = case["n_in"], case["n_out"], case["rank"]
    used = min(case["adapters"], case["requests"])
    weights = used * rank * (n_in + n_out) * es
    if case["kind"] == "adapter_forward":
        return {"bytes": rows * es * (n_in + 2 * n_out) + weights + rows * 4 * (1 + (rank if case["train"] else 0)),
                "flops": 2 * rows * rank * (n_in + n_out)}
    return {"bytes": rows * es * (3 * n_in + n_out) + weights + case["adapters"] * rank * (n_in + n_out) * 4
            + rows * 4 * (1 + rank), "flops": 4 * rows * rank * (n_in + n_out)}


# ------------------------------------------------- the definition in 64 bits
def _kept_exact(rows, cols, p, seed, offset):
    """The dropout factors: 0, or 1 / (1 - p) where an element stays."""
    u64 = np.uint64
    low = u64(0xFFFFFFFF)
    x0 = np.broadcast_to(np.arange(-(-cols // 8), dtype=u64)[None, :], (rows, -(-cols // 8)))
    x1 = np.broadcast_to(np.arange(rows, dtype=u64)[:, None], x0.shape)
    x2, x3 = (np.broadcast_to(u64(v), x0.shape) for v in (offset % 2 ** 32, offset // 2 ** 32 % 2 ** 32))
    for i in range(7):
        k0 = u64((seed % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32)
        k1 = u64((seed // 2 ** 32 % 2 ** 32 + i * 0xBB67AE85) % 2 ** 32)
        p0, p1 = x0 * u64(0xD2511F53), x2 * u64(0xCD9E8D57)
        x0, x1, x2, x3 = (p1 >> u64(32)) ^ x1 ^ k0, p1 & low, (p0 >> u64(32)) ^ x3 ^ k1, p0 & low
    words = np.stack([x0, x1, x2, x3], axis=-1).astype("<u4")
    halves = words.view("<u2").reshape(rows, -1)[:, :cols]
    t = int(round(p * 65536))
    return torch.from_numpy((halves >= t)).to(DEV).double() / (1.0 - t / 65536.0)


def exact(case, seed):
    s = prepare(case, seed)
    wide = lambda t: t.double()  # noqa: E731
    if case["kind"] == "token_loss":
        loss = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
        grad = torch.zeros(case["rows"], case["vocab"], dtype=torch.float64, device=DEV)
        for at in range(0, case["rows"], 256):
            part = slice(at, at + 256)
            rows = torch.nonzero(s["target"][part] >= 0)[:, 0] + at
            z, t = wide(s["logits"][rows]), s["target"][rows]
            w = wide(s["weight"][rows]) if case["weighted"] else torch.ones(len(rows), dtype=torch.float64, device=DEV)
            logp = z - torch.logsumexp(z, 1, keepdim=True)
            index = torch.arange(len(rows), device=DEV)
            loss[rows] = -w * logp[index, t]
            prob = logp.exp()
            prob[index, t] -= 1.0
            grad[rows] = prob * w[:, None]
        return {"loss": loss, "dlogits": grad}
    f = 1.0
    if case["p"] > 0.0:
        f = _kept_exact(case["rows"], case["cols"] if case["kind"] == "dropout" else case["n_in"], case["p"],
                        s["seed"], s["offset"])
    if case["kind"] == "dropout":
        out = wide(s["x"]) * f
        return {"out": out + wide(s["residual"]) if case["residual"] else out}
    x, base = wide(s["x"]) * f, wide(s["base"])
    groups = [(i, torch.nonzero(s["ids"] == i)[:, 0]) for i in range(case["adapters"])]
    if case["kind"] == "adapter_forward":
        y, u = base, torch.zeros(case["rows"], case["rank"], dtype=torch.float64, device=DEV)
        for i, at in groups:
            u[at] = x[at] @ wide(s["a"][i]).T
            y[at] += float(s["scale"][i]) * (u[at] @ wide(s["b"][i]))
        return {"y": y, "u": u} if case["train"] else {"y": y}
    da, db, back = torch.zeros_like(wide(s["a"])), torch.zeros_like(wide(s["b"])), torch.zeros_like(base)
    for i, at in groups:
        c, dy = float(s["scale"][i]), wide(s["dy"][at])
        du = c * (dy @ wide(s["b"][i]).T)
        da[i], db[i] = du.T @ x[at], c * (wide(s["u"][at]).T @ dy)
        back[at] = du @ wide(s["a"][i])
    return {"da": da, "db": db, "dx": base + back * f}
