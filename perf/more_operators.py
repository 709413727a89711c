"""The rest of a tuning step beside a frozen model, as it is timed and compared: norm, preference loss, optimizer.

Subsets of the training data are tried out by tuning a model on each of them.  Beside the adapters' products, dropout and the
token loss (perf/operators.py), a step of that consists of

  layer_norm_forward   h = x + residual, y = (h - mean) / sqrt(var + eps) * gain + bias, or without the mean (rms)
  layer_norm_backward  the gradients of that: dx = base + (what the norm sends back), dgain, dbias
  preference_loss      the loss of pairs of answers (chosen, rejected) by their log ratios, and the gradient of every logit
  adamw                one step of many tensors at once, each subset clipped by its own norm, states in 32 bits or in 8

`run` computes them in elementary torch operations, in 32 bits (the 8-bit states, which a last bit can tip, in 64), or
(with `own`) by the library's entry points.  `exact` computes them in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 256   # elements that share a scale of the 8-bit states

# the linears of one Llama3-8B block, as "inputs x outputs"
LLAMA_BLOCK = "4096x4096,4096x1024,4096x1024,4096x4096,4096x14336,4096x14336,14336x4096"


def listed():
    return [
        # One new token each of 8 requests: the norm in front of a block, with the block before joined to the residual
        # stream.  The smallest serving step, where the launch counts.
        {"name": "norm_serve_8", "kind": "layer_norm_forward", "rows": 8, "cols": 4096, "dtype": "bf16", "rms": True,
         "residual": True, "train": False, "masked": 0.0, "pad": 0},
        # A training step's norm: 16 sequences of 1,024 tokens of a 4096-wide model, with the residual stream.
        {"name": "norm_fwd", "kind": "layer_norm_forward", "rows": 16384, "cols": 4096, "dtype": "bf16", "rms": True,
         "residual": True, "train": True, "masked": 0.0, "pad": 0},
        # The same of GPT-2 small: narrow rows, with mean and bias; padding rows are masked.
        {"name": "norm_fwd_gpt2", "kind": "layer_norm_forward", "rows": 16384, "cols": 768, "dtype": "bf16", "rms": False,
         "residual": True, "train": True, "masked": 0.2, "pad": 0},
        # The backward pass of the 4096-wide norm, with the gradient of the residual stream, padding rows masked.
        {"name": "norm_bwd", "kind": "layer_norm_backward", "rows": 16384, "cols": 4096, "dtype": "bf16", "rms": True,
         "base": True, "masked": 0.2, "pad": 0},
        # The backward pass of GPT-2's norm.
        {"name": "norm_bwd_gpt2", "kind": "layer_norm_backward", "rows": 16384, "cols": 768, "dtype": "bf16",
         "rms": False, "base": True, "masked": 0.0, "pad": 0},
        # The backward pass of a small fp32 model's norm at an odd width.
        {"name": "norm_bwd_f32_odd", "kind": "layer_norm_backward", "rows": 509, "cols": 1001, "dtype": "f32",
         "rms": False, "base": False, "masked": 0.1, "pad": 3},
        # Eight pairs of answers, 2,048 tokens in all, at a large vocabulary; the prompts' tokens are masked.
        {"name": "pairs_128k", "kind": "preference_loss", "rows": 2048, "pairs": 8, "vocab": 128000, "dtype": "bf16",
         "masked": 0.3, "smoothing": 0.0, "weighted": False, "pad": 0},
        # Many short pairs at GPT-2's vocabulary, weighted, labels smoothed, logits in a wider buffer.
        {"name": "pairs_50k", "kind": "preference_loss", "rows": 2041, "pairs": 32, "vocab": 50257, "dtype": "bf16",
         "masked": 0.2, "smoothing": 0.1, "weighted": True, "pad": 7},
        # Three short pairs of a small fp32 model at an odd vocabulary.
        {"name": "pairs_f32_odd", "kind": "preference_loss", "rows": 61, "pairs": 3, "vocab": 5001, "dtype": "f32",
         "masked": 0.0, "smoothing": 0.0, "weighted": False, "pad": 3},
        # Four subsets' adapters of one small layer: the smallest step, where launches count.
        {"name": "step_small", "kind": "adamw", "layers": 1, "linears": "256x1000", "rank": 8, "adapters": 4, "bits": 32,
         "work": False, "clip": True, "gain": 0},
        # Eight subsets' adapters of rank 16 at the seven linears of a block, states in 32 bits.
        {"name": "step_block", "kind": "adamw", "layers": 1, "linears": LLAMA_BLOCK, "rank": 16, "adapters": 8,
         "bits": 32, "work": True, "clip": True, "gain": 4096},
        # The same for four blocks, states in 8 bits.
        {"name": "step_blocks_8bit", "kind": "adamw", "layers": 4, "linears": LLAMA_BLOCK, "rank": 16, "adapters": 8,
         "bits": 8, "work": True, "clip": True, "gain": 4096},
    ]


def _logint(rng, lo, hi, mult=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(mult, v // mult * mult)


def draw(rng):
    kind = rng.choice(("layer_norm_forward", "layer_norm_backward", "layer_norm_backward", "preference_loss",
                       "preference_loss", "adamw", "adamw"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind.startswith("layer_norm"):
        cols = _logint(rng, 33, 16384)
        if rng.random() < 0.5:
            cols = max(64, cols // 64 * 64)
        case = {"kind": kind, "rows": min(_logint(rng, 1, 16384), 60_000_000 // cols), "cols": cols, "dtype": dtype,
                "rms": rng.random() < 0.5, "masked": rng.choice((0.0, 0.2, 0.6)), "pad": -cols % 8 + 8 * rng.randint(0, 2)}
        if kind == "layer_norm_backward":
            return {**case, "base": rng.random() < 0.6}
        return {**case, "residual": rng.random() < 0.6, "train": rng.random() < 0.5}
    if kind == "preference_loss":
        vocab = _logint(rng, 500, 200_000)
        rows = max(2, min(_logint(rng, 2, 4096), 120_000_000 // vocab))
        return {"kind": kind, "rows": rows, "pairs": max(1, min(_logint(rng, 1, 64), rows // 2)), "vocab": vocab,
                "dtype": dtype, "masked": rng.choice((0.0, 0.2, 0.7)), "smoothing": rng.choice((0.0, 0.0, 0.1)),
                "weighted": rng.random() < 0.5, "pad": -vocab % 8}
    rank, adapters = rng.choice((1, 4, 8, 9, 16, 16, 32, 64)), _logint(rng, 1, 64)
    most = max(128, 30_000_000 // (rank * adapters))   # columns of all linears together
    layers, sides, linears = rng.randint(1, 6), 0, []
    for _ in range(rng.randint(1, 7)):
        n_in, n_out = _logint(rng, 64, 14336, 4), _logint(rng, 64, 14336, 4)
        if sides + n_in + n_out <= most // layers or not linears:
            linears.append("%dx%d" % (n_in, n_out))
            sides += n_in + n_out
    return {"kind": kind, "layers": max(1, min(layers, most // sides)), "linears": ",".join(linears), "rank": rank,
            "adapters": max(1, min(adapters, 40_000_000 // (sides * rank))), "bits": rng.choice((8, 32)),
            "work": rng.random() < 0.5, "clip": rng.random() < 0.6, "gain": rng.choice((0, 0, 64, 77, 1001))}


# -------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(np.random.SeedSequence([int(seed), 1607]).generate_state(1)[0]))
    return g


def _rand(g, rows, cols, std, dtype, pad=0):
    """[rows, cols] of N(0, std^2), as a view of rows with `pad` further columns."""
    t = torch.empty(rows, cols + pad, dtype=dtype, device=DEV)
    for at in range(0, rows, 4096):
        part = t[at:at + 4096]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV) * std)
    return t[:, :cols]


def _room(rows, cols, dtype, pad=0):
    return torch.empty(rows, cols + pad, dtype=dtype, device=DEV)[:, :cols]


def _cuts(case, seed):
    """Where the sequences begin in the rows (chosen, rejected, chosen, ...), ragged, each of one token at least."""
    r = np.random.default_rng([int(seed), 53])
    n = 2 * case["pairs"]
    inner = np.sort(r.choice(np.arange(1, case["rows"]), n - 1, replace=False))
    return np.concatenate([[0], inner, [case["rows"]]]).astype(np.int64)


def _slices(case):
    """Elements of a subset's part of each tensor, in the order in which the tensors lie: both factors of every linear, then the
    norms' gains."""
    sides = [int(n) * case["rank"] for pair in case["linears"].split(",") for n in pair.split("x")]
    return sides * case["layers"] + [case["gain"]] * (case["layers"] if case["gain"] > 0 else 0)


def prepare(case, seed):
    g, s = _gen(seed), dict(case)
    f32 = lambda *shape: torch.empty(shape, dtype=torch.float32, device=DEV)  # noqa: E731
    if case["kind"].startswith("layer_norm"):
        rows, cols, pad, dtype = case["rows"], case["cols"], case["pad"], DTYPES[case["dtype"]]
        # a residual stream's values: some columns are far larger than the others, and the mean is not zero
        wide = torch.where(torch.rand(cols, generator=g, device=DEV) < 0.01, 20.0, 1.0)
        x = _rand(g, rows, cols, 1.0, dtype, pad)
        x.copy_(x.float() * wide + 0.3)
        s["gain"] = (1.0 + 0.2 * torch.randn(cols, generator=g, device=DEV)).to(dtype)
        s["bias"] = None if case["rms"] else (0.1 * torch.randn(cols, generator=g, device=DEV)).to(dtype)
        live = torch.rand(rows, generator=g, device=DEV) >= case["masked"]
        s["mask"] = live.to(torch.uint8) if case["masked"] > 0 else None
        s["eps"] = 1e-5
        if case["kind"] == "layer_norm_forward":
            s["x"] = x
            s["residual"] = _rand(g, rows, cols, 2.0, dtype, pad) if case["residual"] else None
            s["h"] = _room(rows, cols, dtype, pad) if case["residual"] else None
            s["y"] = _room(rows, cols, dtype, pad)
            s["mean"], s["rstd"] = (None if case["rms"] or not case["train"] else f32(rows)), (f32(rows) if case["train"] else None)
            return s
        s["h"], s["dy"] = x, _rand(g, rows, cols, 1e-2, dtype, pad)
        s["base"] = _rand(g, rows, cols, 1e-2, dtype, pad) if case["base"] else None
        s["dx"] = _room(rows, cols, dtype, pad)
        # the statistics, as the forward pass left them
        wide_h = x.double()
        mean = torch.zeros(rows, device=DEV, dtype=torch.float64) if case["rms"] else wide_h.mean(1)
        rstd = ((wide_h - mean[:, None]).square().mean(1) + s["eps"]).rsqrt()
        s["mean"], s["rstd"] = (None if case["rms"] else mean.float()), rstd.float()
        s["dgain"], s["dbias"] = f32(cols), (None if case["rms"] else f32(cols))
        if own:   # a workspace that all layers of a width share
            import paper_2405_13954_amd as P
            s["ws"] = torch.empty(max(1, P.logra_layer_norm_ws_size(rows, cols)), dtype=torch.uint8, device=DEV)
        return s
    if case["kind"] == "preference_loss":
        rows, vocab, pairs, dtype = case["rows"], case["vocab"], case["pairs"], DTYPES[case["dtype"]]
        s["logits"] = _rand(g, rows, vocab, 2.5, dtype, case["pad"])
        target = torch.randint(vocab, (rows,), generator=g, device=DEV)
        off = torch.rand(rows, generator=g, device=DEV) < case["masked"]
        s["target"] = torch.where(off, -1, target)
        cuts = _cuts(case, seed)
        s["offsets"] = torch.from_numpy(cuts).to(DEV)
        # the frozen model's sums: near what the tuned model gives
        live = torch.cat([torch.zeros(1, device=DEV), (~off).float().cumsum(0)])[s["offsets"]].diff()
        s["ref"] = -live * (math.log(vocab) + 3.125) + 4.0 * torch.randn(2 * pairs, generator=g, device=DEV)
        s["weight"] = torch.rand(pairs, generator=g, device=DEV) + 0.5 if case["weighted"] else None
        s["beta"] = 0.1
        s["loss"], s["logp"] = f32(pairs), f32(2 * pairs)
        s["dlogits"] = _room(rows, vocab, dtype, case["pad"])
        if own:
            import paper_2405_13954_amd as P
            s["ws"] = torch.empty(max(1, P.logra_preference_loss_ws_size(rows, pairs)), dtype=torch.uint8, device=DEV)
        return s
    lens, n = _slices(case), case["adapters"]
    total = sum(lens) * n
    s["param"] = _rand(g, 1, total, 0.02, torch.float32)[0]
    s["grad"] = _rand(g, 1, total, 1e-3, torch.float32)[0]
    s["work"] = s["param"].to(torch.bfloat16) if case["work"] else None
    m, v = _rand(g, 1, total, 3e-4, torch.float32)[0], _rand(g, 1, total, 1e-3, torch.float32)[0].square()
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        blocks = sum(-(-k // BLOCK) for k in lens) * n
        s["m_scale"] = torch.full((blocks,), 2.0 ** -18, device=DEV)
        s["v_scale"] = torch.full((blocks,), 2.0 ** -30, device=DEV)
        s["m"] = (m * 2.0 ** 18).clamp(-448, 448).to(torch.float8_e4m3fn)
        s["v"] = (v * 2.0 ** 30).clamp(max=57344).to(torch.float8_e5m2)
    s["step"] = torch.full((1,), 9 + int(seed) % 50, dtype=torch.int64, device=DEV)
    s["lr_scale"] = torch.rand(n, generator=g, device=DEV) + 0.5
    s["lr"], s["beta1"], s["beta2"], s["eps"], s["decay"] = 1e-3, 0.9, 0.95, 1e-8, 0.1
    # some subsets' norms are above this and some below
    s["max_norm"] = 1e-3 * math.sqrt(sum(lens)) if case["clip"] else 0.0
    s["norms"] = f32(n) if case["clip"] else None
    s["seed"] = 0x9E3779B97F4A7C15 ^ int(seed)
    if own:   # the list of the tensors, laid out once for all steps
        import paper_2405_13954_amd as P
        tensors, at, block = [], 0, 0
        for i, k in enumerate(lens):
            part, some = slice(at, at + k * n), slice(block, block + -(-k // BLOCK) * n)
            at, block = part.stop, some.stop
            one = {key: s[key][part] for key in ("param", "grad", "m", "v")}
            if case["work"]:
                one["work"] = s["work"][part]
            if case["bits"] == 8:
                one["m_scale"], one["v_scale"] = s["m_scale"][some], s["v_scale"][some]
            tensors.append(P.AdamwTensor(**one, slices=n, decay=not _is_gain(case, i)))
        s["plan"] = P.logra_adamw_plan(tensors, n)
    return s


def _is_gain(case, i):
    """Whether tensor i is a norm's gain, which is not decayed."""
    return i >= 2 * len(case["linears"].split(",")) * case["layers"]


# ------------------------------------------------------------- the plain form
def _plain_norm_forward(s):
    dtype = s["x"].dtype
    live = torch.ones(s["rows"], 1, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"][:, None] != 0
    h = s["x"].float()
    if s["residual"] is not None:
        h = torch.where(live, (h + s["residual"].float()).to(dtype), 0.0)
    c = h.float()
    mean = c.sum(1, keepdim=True) / s["cols"]
    if not s["rms"]:
        c = c - mean
    rstd = 1.0 / torch.sqrt((c * c).sum(1, keepdim=True) / s["cols"] + s["eps"])
    y = c * rstd * s["gain"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    out = {"y": torch.where(live, y, 0.0).to(dtype)}
    if s["residual"] is not None:
        out["h"] = h
    if s["train"]:
        out["rstd"] = torch.where(live, rstd, 0.0)[:, 0]
        if not s["rms"]:
            out["mean"] = torch.where(live, mean, 0.0)[:, 0]
    return out


def _plain_norm_backward(s):
    live = torch.ones(s["rows"], 1, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"][:, None] != 0
    dy = torch.where(live, s["dy"].float(), 0.0)
    c = s["h"].float()
    if not s["rms"]:
        c = c - s["mean"][:, None]
    xh = torch.where(live, c * s["rstd"][:, None], 0.0)
    back = dy * s["gain"].float()
    along = (back * xh).sum(1, keepdim=True) / s["cols"]
    dx = back - xh * along
    if not s["rms"]:
        dx = dx - back.sum(1, keepdim=True) / s["cols"]
    dx = torch.where(live, dx * s["rstd"][:, None], 0.0)
    if s["base"] is not None:
        dx = s["base"].float() + dx
    out = {"dx": dx.to(s["h"].dtype), "dgain": (dy * xh).sum(0)}
    if not s["rms"]:
        out["dbias"] = dy.sum(0)
    return out


def _plain_preference(s):
    z, target, pairs = s["logits"].float(), s["target"], s["pairs"]
    live = target >= 0
    at = target.clamp(min=0)[:, None]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    logp = torch.where(live, (z.gather(1, at) - top - torch.log(total))[:, 0], 0.0)
    sums = torch.cat([torch.zeros(1, dtype=torch.float64, device=DEV), logp.double().cumsum(0)])[s["offsets"]].diff()
    ratio = (sums - s["ref"].double()).view(pairs, 2)
    d = s["beta"] * (ratio[:, 0] - ratio[:, 1])
    soft = lambda t: torch.clamp(t, min=0) + torch.log1p(torch.exp(-t.abs()))  # noqa: E731
    e1 = s["smoothing"]
    weight = torch.ones(pairs, device=DEV) if s["weight"] is None else s["weight"]
    loss = weight * ((1 - e1) * soft(-d) + e1 * soft(d))
    slope = weight * s["beta"] * (e1 - 1 / (1 + torch.exp(d)))
    signed = torch.stack([slope, -slope], 1).view(-1).float()
    row = torch.where(live, signed.repeat_interleave(s["offsets"].diff()), 0.0)[:, None]
    grad = e * (-row / total)
    grad.scatter_add_(1, at, row)
    return {"loss": loss.float(), "logp": sums.float(), "dlogits": grad.to(s["logits"].dtype)}


def _mulhilo(a, b):
    """High and low words of the 64-bit product of 32-bit words held in int64."""
    p = a * b
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _draws(i, part, tensor, step, seed):
    """16 random bits for m and 16 for v of each element: Philox4x32-7 (Salmon et al. 2011) of the counter
    (element / 4, slice, tensor, step), a word for each of four elements, its low half for m."""
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF
    w = [i // 4, part, tensor, torch.zeros_like(i) + step]
    for _ in range(7):
        h0, l0 = _mulhilo(w[0], 0xD2511F53)
        h1, l1 = _mulhilo(w[2], 0xCD9E8D57)
        w = [h1 ^ w[1] ^ k0, l1, h0 ^ w[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    j = i % 4
    word = torch.where(j < 2, torch.where(j == 0, w[0], w[1]), torch.where(j == 2, w[2], w[3]))
    return word & 0xFFFF, word >> 16


def _two_to(k):
    """2^k in 64 bits, exactly."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _to_eight(x, block, members, bits, low, high, draw, least):
    """x (64 bits) as float8 values and the power-of-two scale of each block: the smallest scale that brings the block's
    largest magnitude to 1.75 * 2^high or below; rounded up where the part cut off, in 1/65536 of a step, is above the
    draw.  What is not zero keeps `least` steps of the smallest size at least.  block: the block of each element;
    members: the elements of each block."""
    top = x.abs()[members].amax(1)
    f, e = torch.frexp(top)                                       # top = f 2^e, f in [0.5, 1)
    k = torch.where(top > 0, (e - 1 - high + (f > 0.875)).clamp(-126, 127), 0)
    scale = _two_to(k)
    a = x.abs() / scale[block]
    step = _two_to((torch.frexp(a)[1] - 1).clamp(min=low) - bits)
    whole = torch.floor(a / step)
    whole = whole + ((a / step - whole) * 65536 > draw)
    whole = torch.where(x != 0, whole.clamp(min=least), 0.0)
    return torch.copysign(whole * step, x), scale


def _plain_adamw(s):
    n, dev = s["adapters"], dict(device=DEV)
    lens = torch.tensor(_slices(s), **dev).repeat_interleave(n)                    # of every slice, in order
    starts = lens.cumsum(0) - lens
    part = torch.arange(len(lens), **dev).repeat_interleave(lens)                  # the slice of each element
    mine = part % n                                                                # its subset
    gain = torch.tensor([_is_gain(s, i) for i in range(len(_slices(s)))], **dev)   # not decayed
    wide = torch.float64 if s["bits"] == 8 else torch.float32
    out = {}
    g = s["grad"].to(wide)
    if s["max_norm"] > 0:
        sums = torch.cat([torch.zeros(1, dtype=torch.float64, **dev), s["grad"].double().square().cumsum(0)])
        norm = (sums[starts + lens] - sums[starts]).view(-1, n).sum(0).sqrt()
        out["norms"] = norm.float()
        g = g * torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).to(wide)[mine]
    s["step"] += 1
    t = s["step"].double()
    if s["bits"] == 8:
        i = torch.arange(len(part), **dev) - starts[part]
        per = (lens + BLOCK - 1) // BLOCK
        block = (per.cumsum(0) - per)[part] + i // BLOCK
        of = torch.arange(len(per), **dev).repeat_interleave(per)                  # the slice of each block
        first = starts[of] + BLOCK * (torch.arange(len(of), **dev) - (per.cumsum(0) - per)[of])
        members = torch.minimum(first[:, None] + torch.arange(BLOCK, **dev), (starts + lens)[of][:, None] - 1)
        m, v = s["m"].to(wide) * s["m_scale"].to(wide)[block], s["v"].to(wide) * s["v_scale"].to(wide)[block]
    else:
        m, v = s["m"], s["v"]
    m = s["beta1"] * m + (1 - s["beta1"]) * g
    v = s["beta2"] * v + (1 - s["beta2"]) * (g * g)
    fix1, fix2 = (1 - s["beta1"] ** t).to(wide), (1 - s["beta2"] ** t).to(wide)
    lr = (s["lr"] * s["lr_scale"])[mine]
    decay = torch.where(gain, 0.0, s["decay"])[part // n]
    move = ((m / fix1) / (torch.sqrt(v / fix2) + s["eps"])).float()
    s["param"].copy_(s["param"] * (1 - lr * decay) - lr * move)
    out["param"] = s["param"]
    if s["work"] is not None:
        out["work"] = s["work"].copy_(s["param"])
    if s["bits"] == 8:
        for_m, for_v = _draws(i, mine, part // n, s["step"], s["seed"])
        m, s["m_scale"] = _to_eight(m, block, members, 3, -6, 8, for_m, 0)
        v, s["v_scale"] = _to_eight(v, block, members, 2, -14, 15, for_v, 1)
        s["m"], s["v"] = m.float().to(torch.float8_e4m3fn), v.float().to(torch.float8_e5m2)
        s["m_scale"], s["v_scale"] = s["m_scale"].float(), s["v_scale"].float()
        out.update(m_scale=s["m_scale"], v_scale=s["v_scale"])
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return {**out, "m": s["m"], "v": s["v"]}


# ------------------------------------------------------------- the library
def _own(s):
    import paper_2405_13954_amd as P
    if s["kind"] == "layer_norm_forward":
        P.logra_layer_norm_forward(s["x"], s["y"], gain=s["gain"], bias=s["bias"], eps=s["eps"], rms=s["rms"],
                                   mask=s["mask"], residual=s["residual"], h=s["h"], mean=s["mean"], rstd=s["rstd"])
        return {k: s[k] for k in ("y", "h", "mean", "rstd") if s[k] is not None}
    if s["kind"] == "layer_norm_backward":
        P.logra_layer_norm_backward(s["h"], s["dy"], s["rstd"], mean=s["mean"], gain=s["gain"], rms=s["rms"],
                                    mask=s["mask"], dx=s["dx"], base=s["base"], dgain=s["dgain"], dbias=s["dbias"],
                                    ws=s["ws"])
        return {k: s[k] for k in ("dx", "dgain", "dbias") if s[k] is not None}
    if s["kind"] == "preference_loss":
        P.logra_preference_loss(s["logits"], s["target"], s["offsets"], s["logp"], loss=s["loss"], dlogits=s["dlogits"],
                                ref=s["ref"], weight=s["weight"], beta=s["beta"], smoothing=s["smoothing"], ws=s["ws"])
        return {k: s[k] for k in ("loss", "logp", "dlogits")}
    P.logra_adamw_step(s["plan"], s["step"], s["lr"], beta1=s["beta1"], beta2=s["beta2"], eps=s["eps"],
                       weight_decay=s["decay"], max_norm=s["max_norm"], lr_scale=s["lr_scale"], norms=s["norms"],
                       seed=s["seed"])
    return {k: s[k] for k in ("param", "work", "m", "v", "m_scale", "v_scale", "norms") if s.get(k) is not None}


def run(s):
    if own:
        return _own(s)
    return {"layer_norm_forward": _plain_norm_forward, "layer_norm_backward": _plain_norm_backward,
            "preference_loss": _plain_preference, "adamw": _plain_adamw}[s["kind"]](s)


# -------------------------------------------------------------------- floors
def work(case):
    if case["kind"] == "adamw":
        n = sum(_slices(case)) * case["adapters"]
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (12 + state + (2 if case["work"] else 0)), "flops": 20 * n}
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "preference_loss":
        n = case["rows"] * case["vocab"]   # masked rows are written, and not read
        return {"bytes": n * es * (2 - case["masked"]) + case["rows"] * 8 + case["pairs"] * 32, "flops": 6 * n}
    n, live = case["rows"] * case["cols"], 1 - case["masked"]
    if case["kind"] == "layer_norm_forward":
        joined = 2 if case["residual"] else 1
        return {"bytes": n * es * (live * joined + joined) + (8 * case["rows"] if case["train"] else 0) + 2 * case["cols"] * es,
                "flops": 6 * n}
    return {"bytes": n * es * (2 * live + 1 + (1 if case["base"] else 0)) + 8 * case["rows"]
            + case["cols"] * (es + (4 if case["rms"] else 8)), "flops": 10 * n}


# ------------------------------------------------- the definition in 64 bits
def _exact_norm(case, s):
    dtype = DTYPES[case["dtype"]]
    rows = torch.arange(case["rows"], device=DEV) if s["mask"] is None else torch.nonzero(s["mask"])[:, 0]
    gain = s["gain"].double()
    full = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)  # noqa: E731
    if case["kind"] == "layer_norm_forward":
        h = s["x"][rows].double()
        if case["residual"]:
            h = (h + s["residual"][rows].double()).to(dtype).double()   # the norm is that of the stored sum
        mean = torch.zeros_like(h[:, :1]) if case["rms"] else h.mean(1, keepdim=True)
        rstd = (torch.mean((h - mean) ** 2, 1, keepdim=True) + s["eps"]) ** -0.5
        y = full(case["rows"], case["cols"])
        y[rows] = (h - mean) * rstd * gain + (0 if s["bias"] is None else s["bias"].double())
        out = {"y": y}
        if case["residual"]:
            out["h"] = full(case["rows"], case["cols"])
            out["h"][rows] = h
        if case["train"]:
            for key, value in (("rstd", rstd), ("mean", mean)):
                if s[key] is not None:
                    out[key] = full(case["rows"])
                    out[key][rows] = value[:, 0]
        return out
    dy, rstd = s["dy"][rows].double(), s["rstd"][rows].double()[:, None]
    unit = s["h"][rows].double() * rstd
    if not case["rms"]:
        unit = unit - s["mean"][rows].double()[:, None] * rstd
    c = dy * gain
    inner = c - unit * torch.mean(c * unit, 1, keepdim=True)
    if not case["rms"]:
        inner -= torch.mean(c, 1, keepdim=True)
    dx = full(case["rows"], case["cols"]) if s["base"] is None else s["base"].double()
    dx[rows] += rstd * inner
    out = {"dx": dx, "dgain": torch.sum(dy * unit, 0)}
    return out if case["rms"] else {**out, "dbias": torch.sum(dy, 0)}


def _exact_preference(case, s):
    cuts, slopes, losses, sums = s["offsets"].tolist(), [], [], []
    logp = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
    norm = torch.zeros_like(logp)
    rows = torch.nonzero(s["target"] >= 0)[:, 0]
    for some in rows.split(256):
        z = s["logits"][some].double()
        norm[some] = torch.logsumexp(z, 1)
        logp[some] = z[torch.arange(len(some), device=DEV), s["target"][some]] - norm[some]
    logp = logp.cpu().numpy()
    for i in range(case["pairs"]):
        a, b = (math.fsum(logp[cuts[j]:cuts[j + 1]]) for j in (2 * i, 2 * i + 1))
        sums += [a, b]
        d = s["beta"] * (a - float(s["ref"][2 * i]) - b + float(s["ref"][2 * i + 1]))
        w, e = (1.0 if s["weight"] is None else float(s["weight"][i])), case["smoothing"]
        losses.append(w * ((1 - e) * np.logaddexp(0.0, -d) + e * np.logaddexp(0.0, d)))
        up = 1 / (1 + math.exp(-d))
        slopes += [w * s["beta"] * (e * up - (1 - e) * (1 - up))] * 2
        slopes[-1] *= -1
    each = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
    for j, f in enumerate(slopes):
        each[cuts[j]:cuts[j + 1]] = f
    grad = torch.zeros(case["rows"], case["vocab"], dtype=torch.float64, device=DEV)
    for some in rows.split(256):
        p = torch.exp(s["logits"][some].double() - norm[some, None])
        p[torch.arange(len(some), device=DEV), s["target"][some]] -= 1
        grad[some] = -each[some, None] * p
    wide = lambda v: torch.tensor(v, dtype=torch.float64, device=DEV)  # noqa: E731
    return {"loss": wide(losses), "logp": wide(sums), "dlogits": grad}


def _exact_bits(count, part, tensor, step, seed):
    """[2, count]: the 16 bits drawn for m and for v of a slice's elements."""
    quads = -(-count // 4)
    low = 0xFFFFFFFF
    c = [torch.arange(quads, device=DEV)] + [torch.full((quads,), v, dtype=torch.int64, device=DEV) for v in (part, tensor, step & low)]
    for r in range(7):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        k0, k1 = ((seed + r * 0x9E3779B9) & low, ((seed >> 32) + r * 0xBB67AE85) & low)
        c = [((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low]
    words = torch.stack(c, 1).reshape(-1)[:count]
    return torch.stack([words % 65536, words // 65536])


def _exact_eight(x, draw, mantissa, floor_exp, top_exp, never_zero):
    """One slice's states in 8 bits: (values before the scale, scales)."""
    pad = -len(x) % BLOCK
    powers = torch.tensor([2.0 ** j for j in range(-300, 301)], dtype=torch.float64, device=DEV)
    exponent = lambda t: torch.searchsorted(powers, t, right=True) - 301  # noqa: E731   (2^e <= t < 2^(e + 1))
    a = torch.nn.functional.pad(x.abs(), (0, pad)).view(-1, BLOCK)
    top = a.amax(1, keepdim=True)
    k = exponent(top)
    k = torch.where(top > 0, (k - top_exp + (top / powers[k.clamp(min=-300) + 300] > 1.75)).clamp(-126, 127), 0)
    scale = powers[k + 300]
    a = a / scale
    ulp = powers[exponent(a).clamp(min=floor_exp) - mantissa + 300]
    n = torch.floor(a / ulp)
    n = n + (a / ulp - n > torch.nn.functional.pad(draw, (0, pad)).view(-1, BLOCK) / 65536)
    if never_zero:
        n = torch.where((a > 0) & (n == 0), 1.0, n)
    return (n * ulp).view(-1)[:len(x)] * torch.sign(x), scale[:, 0]


def _exact_adamw(case, s):
    n, lens = case["adapters"], _slices(case)
    at = np.concatenate([[0], np.cumsum(np.repeat(lens, n))])
    grad = [s["grad"][at[i]:at[i + 1]].double() for i in range(len(at) - 1)]
    norms = [math.sqrt(sum(float(torch.dot(g, g)) for g in grad[a::n])) for a in range(n)]
    t = int(s["step"]) + 1
    got = {k: [] for k in ("param", "m", "v", "m_scale", "v_scale")}
    block = 0
    for i, g in enumerate(grad):
        a, some = i % n, slice(int(at[i]), int(at[i + 1]))
        if 0 < s["max_norm"] < norms[a]:
            g = g * (s["max_norm"] / norms[a])
        m, v = s["m"][some].double(), s["v"][some].double()
        if case["bits"] == 8:
            here = slice(block, block + -(-len(g) // BLOCK))
            block = here.stop
            m = m * s["m_scale"][here].double().repeat_interleave(BLOCK)[:len(g)]
            v = v * s["v_scale"][here].double().repeat_interleave(BLOCK)[:len(g)]
        m = s["beta1"] * m + (1 - s["beta1"]) * g
        v = s["beta2"] * v + (1 - s["beta2"]) * g ** 2
        lr = s["lr"] * float(s["lr_scale"][a])
        p = s["param"][some].double()
        if not _is_gain(case, i // n):
            p = p - lr * s["decay"] * p
        p = p - lr * (m / (1 - s["beta1"] ** t)) / (torch.sqrt(v / (1 - s["beta2"] ** t)) + s["eps"])
        if case["bits"] == 8:
            bits = _exact_bits(len(g), a, i // n, t, s["seed"])
            m, scale = _exact_eight(m, bits[0], 3, -6, 8, False)
            got["m_scale"].append(scale)
            v, scale = _exact_eight(v, bits[1], 2, -14, 15, True)
            got["v_scale"].append(scale)
        for key, value in (("param", p), ("m", m), ("v", v)):
            got[key].append(value)
    out = {k: torch.cat(v) for k, v in got.items() if v}
    if case["work"]:
        out["work"] = out["param"]
    return {**out, "norms": torch.tensor(norms, dtype=torch.float64, device=DEV)} if case["clip"] else out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("layer_norm"):
        return _exact_norm(case, s)
    return _exact_preference(case, s) if case["kind"] == "preference_loss" else _exact_adamw(case, s)
