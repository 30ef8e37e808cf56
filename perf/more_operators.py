"""Rotary positions of several axes, norms of heads with them, attention in a window and behind a shared prefix, as measurable cases.

A case is a dict of plain values.  Four kinds:

  axes    rotary positions of up to three axes (frame, row, column) on the q and k slices of a QKV layer's output.
  norm    the norm of every head of q and k and such positions behind it.
  window  attention over packed sequences in a sliding window, a few first tokens always visible.
  prefix  attention over packed sequences that share their first keys.

`own` false: elementary torch operations in 32 bits (angles in 64).  `own` true: the calls of this package.  Sizes: the
image and video DiT blocks of this repository (16 heads of 72, 8192 and 32768 tokens, captions of 120), and generic
grouped heads of 128 channels.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


# ---- cases -----------------------------------------------------------------------------------------------------

def _positions(name, kind, grid, heads, kv_heads, head_dim, sections, pairing, dtype, norm=None):
    """grid: sizes of the axes, the last the fastest ("2x64x64").  sections: pairs of every axis ("18,18"), together at most head_dim / 2."""
    case = {"name": name, "kind": kind, "grid": grid, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "sections": sections, "pairing": pairing, "dtype": dtype}
    return case if norm is None else {**case, "norm": norm}


def _window(name, sequences, queries, keys, ragged, heads, kv_heads, head_dim, causal, left, right, sinks, dtype):
    """keys 0: every sequence has as many keys as queries.  ragged: lengths up to the given ones."""
    return {"name": name, "kind": "window", "sequences": sequences, "queries": queries, "keys": keys, "ragged": ragged,
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "left": left, "right": right,
            "sinks": sinks, "dtype": dtype}


def _prefix(name, sequences, prefix, queries, keys, ragged, heads, kv_heads, head_dim, causal, dtype):
    return {"name": name, "kind": "prefix", "sequences": sequences, "prefix": prefix, "queries": queries, "keys": keys,
            "ragged": ragged, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "dtype": dtype}


def listed():
    return [
        # one small picture among text, half of the head turned: latency
        _positions("axes_thumbnail", "axes", "1x5x7", 32, 8, 128, "8,12,12", "neighbours", "bf16"),
        # q and k of an image DiT pair, every axis in halves of its own
        _positions("axes_image", "axes", "2x64x64", 16, 16, 72, "18,18", "axis_halves", "f16"),
        # q and k of a video DiT's block
        _positions("axes_video", "axes", "32x32x32", 16, 16, 72, "8,14,14", "halves", "f16"),
        # a few new tokens, grouped heads
        _positions("norm_tokens", "norm", "16", 32, 8, 128, "64", "halves", "bf16", "rms"),
        # an odd number of tokens, mean and variance with bias, a part of the head turned
        _positions("norm_ragged", "norm", "3x41x59", 20, 4, 96, "4,10,10", "axis_halves", "bf16", "layer"),
        # q and k of a video DiT's block
        _positions("norm_video", "norm", "32x32x32", 16, 16, 72, "8,14,14", "neighbours", "f16", "rms"),
        # self-attention of a video DiT pair to neighbouring tokens, the first row always visible
        _window("window_video", 2, 16384, 0, False, 16, 16, 72, False, 1024, 1024, 32, "f16"),
        # prompts of different lengths, causal, grouped heads
        _window("window_prompts", 6, 8192, 0, True, 32, 8, 128, True, 1023, 0, 4, "bf16"),
        # one new token per sequence over long keys of different lengths
        _window("window_tokens", 48, 1, 32768, True, 32, 8, 128, True, 4095, 0, 4, "f16"),
        # single tokens behind one long prompt
        _prefix("prefix_tokens", 64, 8192, 1, 700, True, 32, 8, 128, True, "bf16"),
        # a few sequences of drafted tokens behind a very long one, odd lengths
        _prefix("prefix_drafts", 5, 30011, 7, 301, True, 16, 2, 64, True, "f16"),
        # images of one caption: all see its tokens and their own
        _prefix("prefix_images", 6, 300, 4096, 0, False, 16, 16, 72, False, "f16"),
    ]


def _numbers(text):
    return [int(n) for n in text.replace("x", ",").split(",")]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_positions(rng, kind, dtype):
    kv_heads = rng.choice((1, 2, 8, 16))
    heads = kv_heads * rng.choice((1, 2, 4))
    head_dim = rng.choice((64, 72, 96, 128))
    most = min(32768, 32768 * 2 * 1152 // ((heads + kv_heads) * head_dim))
    axes = rng.choice((1, 2, 3))
    tokens = _log_int(rng, 1, most)
    if axes == 1:
        grid = [tokens]
    else:
        side = max(1, math.isqrt(min(tokens, 4096)))
        row = _log_int(rng, max(1, side // 3), side)
        grid = [side, row] if axes == 2 else [max(1, tokens // (side * row)), side, row]
    pairs = rng.choice((head_dim // 2, head_dim // 2, head_dim // 4, 24))
    cuts = sorted(rng.sample(range(1, pairs), axes - 1))
    sections = [b - a for a, b in zip([0] + cuts, cuts + [pairs])]
    case = {"kind": kind, "grid": "x".join(map(str, grid)), "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "sections": ",".join(map(str, sections)), "pairing": rng.choice(("halves", "neighbours", "axis_halves")), "dtype": dtype}
    return case if kind == "axes" else {**case, "norm": rng.choice(("rms", "rms", "layer"))}


def draw(rng):
    kind = rng.choice(("axes", "norm", "window", "window", "prefix", "prefix"))
    dtype = rng.choice(("f16", "bf16"))
    if kind in ("axes", "norm"):
        return _draw_positions(rng, kind, dtype)
    kv_heads = rng.choice((1, 2, 8))
    heads = kv_heads * rng.choice((1, 2, 4))
    head_dim = rng.choice((64, 72, 80, 96, 128))
    sequences = _log_int(rng, 1, 64)
    case = {"kind": kind, "sequences": sequences, "ragged": rng.random() < 0.7, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "dtype": dtype}
    room = 60_000_000_000 // (heads * head_dim)           # pairs of a query and a key
    if kind == "window":
        left, sinks = _log_int(rng, 16, 4096), rng.choice((0, 1, 4, 17, 100))
        if rng.random() < 0.5:       # whole sequences, to both sides or backwards
            causal = rng.random() < 0.5
            right = 0 if causal else rng.choice((left, left, left // 2))
            most = min(room // (left + right + sinks + 1), 32768 * 1152 // (heads * head_dim)) // sequences
            queries, keys = min(_log_int(rng, 16, 16384), max(16, most)), 0
        else:                        # a few new tokens over long keys
            queries, keys, causal, right = rng.choice((1, 1, 2, 5, 64)), _log_int(rng, 256, 32768), True, 0
            keys = min(keys, 1_500_000 // sequences * 8 // kv_heads)
        return {**case, "queries": queries, "keys": keys, "causal": causal, "left": left, "right": right, "sinks": sinks}
    prefix = _log_int(rng, 16, 32768)
    if rng.random() < 0.4:           # whole sequences behind it
        most = max(16, min(room // (sequences * prefix), math.isqrt(room // sequences), 32768 * 1152 // (sequences * heads * head_dim)))
        queries, keys, causal = min(_log_int(rng, 16, 4096), most), 0, rng.random() < 0.5
    else:                            # a few new tokens
        queries, keys, causal = rng.choice((1, 1, 2, 5, 16)), _log_int(rng, 1, 2048) + 16, True
        prefix = min(prefix, room // (sequences * queries))
    return {**case, "prefix": prefix, "queries": queries, "keys": keys, "causal": causal}


def _lengths(case):
    """Queries and keys of every sequence; the longest is the case's own, the others spread over their logarithm."""
    rng = random.Random(case["sequences"] * 7919 + case["queries"] * 31 + case["keys"])
    top = case["keys"] or case["queries"]
    n = case["sequences"]
    long = [top] + [_log_int(rng, max(1, top // 16), top) if case["ragged"] else top for _ in range(n - 1)]
    rng.shuffle(long)
    return ([case["queries"]] * n, long) if case["keys"] else (long, long)


def _seen(case, n, m):
    """(pairs of a query and a key that it sees, keys that any query sees) of a sequence in a window."""
    i = torch.arange(m - n, m)
    last = torch.clamp(i, max=m - 1) if case["causal"] else torch.full_like(i, m - 1)
    hi = torch.minimum(i + case["right"], last)                       # the last key in the window
    lo = torch.clamp(i - case["left"], min=0)
    window = torch.clamp(hi - lo + 1, min=0)
    sinks = torch.clamp(last + 1, min=0, max=case["sinks"])
    both = torch.clamp(torch.minimum(sinks, hi + 1) - lo, min=0) * (window > 0)
    widest = int(hi.max()) - int(lo.min()) + 1
    return int((window + sinks - both).sum()), min(m, max(widest, 0) + min(case["sinks"], int(lo.min())))


def work(case):
    kind = case["kind"]
    D, H, G = case["head_dim"], case["heads"], case["kv_heads"]
    if kind in ("axes", "norm"):
        sections = _numbers(case["sections"])
        T, R = math.prod(_numbers(case["grid"])), 2 * sum(sections)
        values = T * (H + G) * D
        vectors = 4 * D * (4 if case.get("norm") == "layer" else 2) if kind == "norm" else 0
        return {"bytes": 4 * values + 4 * T * len(sections) + 2 * R + vectors,
                "flops": 3 * T * (H + G) * R + (4 * values if kind == "norm" else 0)}
    lq, lk = _lengths(case)
    if kind == "window":
        seen = [_seen(case, n, m) for n, m in zip(lq, lk)]
        pairs, keys = sum(p for p, _ in seen), sum(k for _, k in seen)
    else:
        pairs = sum(n * (case["prefix"] + m) - (n * (n - 1) // 2 if case["causal"] else 0) for n, m in zip(lq, lk))
        keys = case["prefix"] + sum(lk)
    return {"bytes": 4 * sum(lq) * H * D + 4 * keys * G * D + 8 * len(lq) + 8, "flops": 4 * pairs * H * D}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _pairs(sections, pairing):
    """Channels of the first and of the second of every pair."""
    n = sum(sections)
    i = torch.arange(n, device="cuda")
    if pairing == "halves":
        return i, i + n
    if pairing == "neighbours":
        return 2 * i, 2 * i + 1
    size = torch.tensor(sections, device="cuda")
    first = (torch.cumsum(size, 0) - size).repeat_interleave(size)
    return i + first, i + first + size.repeat_interleave(size)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype, kind = TYPES[case["dtype"]], case["kind"]
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    s = {"case": case, "dtype": dtype}

    def heads(T, n, spread=False):
        x = torch.randn(T, n, D, generator=g, device="cuda")
        if spread:                   # tokens and channels of different size, as in front of a norm
            x = x * torch.exp(torch.randn(T, 1, 1, generator=g, device="cuda")) * torch.exp(0.5 * torch.randn(D, generator=g, device="cuda"))
        return x.to(dtype)

    if kind in ("axes", "norm"):
        grid, sections = _numbers(case["grid"]), _numbers(case["sections"])
        T, axes = math.prod(grid), len(sections)
        qkv = heads(T, H + 2 * G, kind == "norm")
        s["q"], s["k"] = qkv[:, :H], qkv[:, H:H + G]          # slices of the QKV layer's output
        at = torch.cartesian_prod(*(torch.arange(n, device="cuda") for n in grid)).reshape(T, -1)
        first = torch.randint(0, 2000, (axes, 1), generator=g, device="cuda")
        s["positions"] = (at.t()[-axes:] + first).to(torch.int32).contiguous()       # a grid somewhere in its space
        s["inv_freq"] = torch.cat([10000.0 ** (torch.arange(n, device="cuda", dtype=torch.float64) / -n) for n in sections]).float()
        s["sections"] = sections
        s["axis"] = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], device="cuda")
        s["pairs"] = _pairs(sections, case["pairing"])
        if kind == "norm":
            s["weights"] = [1 + 0.2 * torch.randn(D, generator=g, device="cuda") for _ in range(2)]
            s["biases"] = [0.1 * torch.randn(D, generator=g, device="cuda") if case["norm"] == "layer" else None for _ in range(2)]
        return s
    lq, lk = _lengths(case)
    s["lq"], s["lk"] = lq, lk
    s["cu_q"], s["cu_k"] = (torch.tensor([0] + l, device="cuda").cumsum(0).to(torch.int32) for l in (lq, lk))
    if case["keys"]:
        s["q"] = heads(sum(lq), H)
        kv = heads(sum(lk), 2 * G)
        s["k"], s["v"] = kv[:, :G], kv[:, G:]
    else:
        qkv = heads(sum(lq), H + 2 * G)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
    if kind == "prefix":
        kv = heads(case["prefix"], 2 * G)
        s["prefix_k"], s["prefix_v"] = kv[:, :G], kv[:, G:]
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------

def _plain_turn(t, s):
    """t in 32 bits."""
    angle = (s["positions"][s["axis"]].t().double() * s["inv_freq"].double()).unsqueeze(1)
    cos, sin = angle.cos().float(), angle.sin().float()
    first, second = s["pairs"]
    a, b = t[..., first], t[..., second]
    out = t.clone()
    out[..., first], out[..., second] = a * cos - b * sin, b * cos + a * sin
    return out


def _plain_norm(x, weight, bias, case):
    t = x.float()
    if case["norm"] == "layer":
        t = t - t.mean(-1, keepdim=True)
    t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * weight
    return t if bias is None else t + bias


def _plain_rows(scores, v):
    """softmax(scores [H,n,m], hidden ones -inf) v [m,G,D] in 32 bits: [n,H,D], zeros for a row that sees nothing."""
    H, n, m = scores.shape
    G, D = v.shape[1:]
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.bmm(p.reshape(G, -1, m), v.transpose(0, 1).contiguous()).reshape(H, n, D)
    return torch.where(total > 0, out / total, 0.0).transpose(0, 1)


def _plain_scores(q, k):
    n, H, D = q.shape
    m, G = k.shape[:2]
    q = q.transpose(0, 1).reshape(G, -1, D)                                          # a group's heads one after another
    return torch.bmm(q, k.permute(1, 2, 0).contiguous()).reshape(H, n, m) / math.sqrt(D)


def _plain_block(q, k, v, first, case, m):
    """Queries at positions first .. of a sequence with m keys, to the keys that any of them sees."""
    n = q.shape[0]
    i = torch.arange(first, first + n, device=q.device)[:, None]
    lo, hi = max(0, first - case["left"]), max(0, min(m, first + n + case["right"]))
    sinks = min(case["sinks"], lo, m)
    j = torch.cat((torch.arange(sinks, device=q.device), torch.arange(lo, max(lo, hi, min(case["sinks"], m)), device=q.device)))
    seen = ((j >= i - case["left"]) & (j <= i + case["right"])) | (j < case["sinks"])
    if case["causal"]:
        seen = seen & (j <= i)
    if j.numel() == 0:
        return torch.zeros_like(q)
    return _plain_rows(_plain_scores(q.float(), k[j].float()).masked_fill(~seen, -math.inf), v[j].float()).to(q.dtype)


def _plain_window(q, k, v, case):
    """One sequence, in blocks of queries that leave most of the keys that they do not see."""
    n, m = q.shape[0], k.shape[0]
    step = max(256, case["left"] + case["right"])
    return torch.cat([_plain_block(q[i:i + step], k, v, i + m - n, case, m) for i in range(0, n, step)])


def _plain_behind(q, k, v, scores, prefix_v, causal):
    """One sequence, its scores with the prefix computed for all before."""
    n, m = q.shape[0], k.shape[0]
    its = _plain_scores(q.float(), k.float())
    if causal:
        hidden = torch.arange(m, device=q.device) > torch.arange(n, device=q.device)[:, None] + (m - n)
        its = its.masked_fill(hidden, -math.inf)
    return _plain_rows(torch.cat((scores, its), -1), torch.cat((prefix_v, v.float()))).to(q.dtype)


def _plain(s):
    case = s["case"]
    if case["kind"] == "axes":
        return tuple(_plain_turn(x.float(), s).to(s["dtype"]) for x in (s["q"], s["k"]))
    if case["kind"] == "norm":
        return tuple(_plain_turn(_plain_norm(x, w, b, case), s).to(s["dtype"])
                     for x, w, b in zip((s["q"], s["k"]), s["weights"], s["biases"]))
    parts = zip(s["q"].split(s["lq"]), s["k"].split(s["lk"]), s["v"].split(s["lk"]))
    if case["kind"] == "window":
        return torch.cat([_plain_window(q, k, v, case) for q, k, v in parts])
    prefix_k, prefix_v = s["prefix_k"].float(), s["prefix_v"].float()
    scores = _plain_scores(s["q"].float(), prefix_k).split(s["lq"], 1)
    return torch.cat([_plain_behind(q, k, v, its, prefix_v, case["causal"]) for (q, k, v), its in zip(parts, scores)])


def run(state):
    if not own:
        return _plain(state)
    import paper_2406_02540_amd as vq
    s, case = state, state["case"]
    if case["kind"] == "axes":
        return vq.vq_rotary_axes(s["q"], s["k"], s["positions"], s["inv_freq"], s["sections"], pairing=case["pairing"])
    if case["kind"] == "norm":
        return vq.vq_norm_rotary(s["q"], s["k"], *s["weights"], *s["biases"], norm=case["norm"], eps=1e-6, positions=s["positions"],
                                 inv_freq=s["inv_freq"], sections=s["sections"], pairing=case["pairing"])
    if case["kind"] == "window":
        return vq.vq_attention_window(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], case["left"], case["right"], sinks=case["sinks"],
                                      causal=case["causal"])
    return vq.vq_attention_prefix(s["q"], s["prefix_k"], s["prefix_v"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=case["causal"])


# ---- the definitions in 64 bits --------------------------------------------------------------------------------

def _exact_positions(s):
    """Axis by axis, pairs as complex numbers."""
    case = s["case"]
    outs = []
    for n, x in enumerate((s["q"], s["k"])):
        y = x.double()
        if case["kind"] == "norm":
            if case["norm"] == "layer":
                y = (y - y.mean(-1, keepdim=True)) * (y.var(-1, correction=0, keepdim=True) + 1e-6) ** -0.5
            else:
                y = y * (y.pow(2).mean(-1, keepdim=True) + 1e-6) ** -0.5
            y = y * s["weights"][n].double()
            if s["biases"][n] is not None:
                y = y + s["biases"][n].double()
        y = y.clone()
        total, at = sum(s["sections"]), 0
        for axis, size in enumerate(s["sections"]):
            if case["pairing"] == "neighbours":
                a, b = slice(2 * at, 2 * (at + size), 2), slice(2 * at + 1, 2 * (at + size), 2)
            elif case["pairing"] == "halves":
                a, b = slice(at, at + size), slice(total + at, total + at + size)
            else:
                a, b = slice(2 * at, 2 * at + size), slice(2 * at + size, 2 * (at + size))
            angle = torch.outer(s["positions"][axis].double(), s["inv_freq"][at:at + size].double())
            z = torch.complex(y[..., a], y[..., b]) * torch.polar(torch.ones_like(angle), angle)[:, None]
            y[..., a], y[..., b] = z.real, z.imag
            at += size
        outs.append(y)
    return tuple(outs)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("axes", "norm"):
        return _exact_positions(s)
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    out = torch.zeros_like(q)
    share, scale = case["heads"] // case["kv_heads"], case["head_dim"] ** -0.5
    at, bt = 0, 0
    for n, m in zip(s["lq"], s["lk"]):
        j = torch.arange(m, device=q.device).unsqueeze(0)
        i = torch.arange(n, device=q.device).unsqueeze(1) + m - n
        hide = (j > i) if case["causal"] else torch.zeros(n, m, dtype=torch.bool, device=q.device)
        if case["kind"] == "window":
            hide = hide | (((j - i > case["right"]) | (i - j > case["left"])) & (j >= case["sinks"]))
        for h in range(case["heads"]):
            kh, vh = k[bt:bt + m, h // share], v[bt:bt + m, h // share]
            w = (q[at:at + n, h] @ kh.T * scale).masked_fill(hide, -math.inf)
            if case["kind"] == "prefix":
                w = torch.cat((q[at:at + n, h] @ s["prefix_k"][:, h // share].double().T * scale, w), 1)
                vh = torch.cat((s["prefix_v"][:, h // share].double(), vh))
            out[at:at + n, h] = torch.nan_to_num(torch.softmax(w, 1)) @ vh
        at, bt = at + n, bt + m
    return out
