"""Microscaled 4-bit layers, rotary positions and attention, as measurable cases.

A case is a dict of plain values.  Five kinds:

  codes      activations to microscaled 4-bit codes (e2m1, one power-of-two scale per 32 channels) and read back.
  product    the GEMM on such codes, both operands quantized before.
  layer      quantizer and GEMM in one call, weights quantized before, as a module keeps them.
  rotary     rotary positions on the q and k slices of a QKV layer's output.
  attention  softmax attention over packed sequences of different lengths, grouped heads, causal or not.

`own` false: elementary torch operations in 32 bits (the angles of rotary positions in 64).  `own` true: the calls of
this package.  Sizes: the image and video DiT layers of this repository (hidden 1152 in 16 heads, MLP 4608, 8192 and
32768 tokens, text of 4096 channels), and generic grouped heads of 128 channels.
"""
from __future__ import annotations

import math
import random

import torch

own = False

HIDDEN, MLP, TEXT = 1152, 4608, 4096
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


# ---- cases -----------------------------------------------------------------------------------------------------

def _codes(name, M, K, dtype, balanced):
    return {"name": name, "kind": "codes", "M": M, "K": K, "dtype": dtype, "balanced": balanced}


def _gemm(name, kind, M, K, N, dtype, balanced=False):
    return {"name": name, "kind": kind, "M": M, "K": K, "N": N, "dtype": dtype, "balanced": balanced}


def _rotary(name, T, heads, kv_heads, head_dim, rot_dim, interleaved, far, dtype):
    return {"name": name, "kind": "rotary", "T": T, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "rot_dim": rot_dim, "interleaved": interleaved, "far": far, "dtype": dtype}


def _attention(name, sequences, queries, keys, ragged, heads, kv_heads, head_dim, causal, dtype):
    """keys 0: every sequence has as many keys as queries.  ragged: lengths up to the given ones."""
    return {"name": name, "kind": "attention", "sequences": sequences, "queries": queries, "keys": keys, "ragged": ragged,
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "dtype": dtype}


def listed():
    return [
        # a few caption tokens in the other 16-bit type: one short launch
        _codes("codes_caption", 77, 1184, "bf16", False),
        # MLP output layer's input of an image DiT pair, with its balancing mask: bound by memory
        _codes("codes_image_fc2", 8192, MLP, "f16", True),
        # sizes that no tile divides, odd N
        _gemm("product_ragged", "product", 1001, 1184, 2821, "bf16"),
        # MLP input layer of a video DiT: the largest product
        _gemm("product_video_fc1", "product", 32768, HIDDEN, MLP, "f16"),
        # one token through a QKV layer: latency
        _gemm("layer_one_token", "layer", 1, HIDDEN, 3 * HIDDEN, "f16"),
        # cross-attention k/v of a prompt pair: few tokens, long K
        _gemm("layer_text_kv", "layer", 240, TEXT, 2 * HIDDEN, "f16", True),
        # single tokens far into long contexts, grouped heads, half of the head rotated, neighbouring pairs
        _rotary("rotary_far_tokens", 16, 32, 8, 128, 64, True, True, "bf16"),
        # q and k of a video DiT's block
        _rotary("rotary_video", 32768, 16, 16, 72, 72, False, False, "f16"),
        # self-attention of an image DiT pair
        _attention("attention_image", 2, 4096, 0, False, 16, 16, 72, False, "f16"),
        # cross-attention of a video DiT pair to its captions
        _attention("attention_captions", 2, 16384, 120, True, 16, 16, 72, False, "f16"),
        # prompts of different lengths, causal, grouped heads
        _attention("attention_prompts", 6, 8192, 0, True, 32, 8, 128, True, "bf16"),
        # one new token per sequence over long keys of different lengths
        _attention("attention_tokens", 16, 1, 32768, True, 32, 8, 128, True, "f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_k(rng):
    if rng.random() < 0.4:
        return rng.choice((HIDDEN, TEXT, MLP))
    return max(32, _log_int(rng, 64, MLP) // 32 * 32)


def draw(rng):
    kind = rng.choice(("codes", "product", "layer", "rotary", "attention", "attention"))
    dtype = rng.choice(("f16", "bf16"))
    if kind == "codes":
        return {"kind": kind, "M": _log_int(rng, 1, 8192), "K": _draw_k(rng), "dtype": dtype, "balanced": rng.random() < 0.5}
    if kind in ("product", "layer"):
        K = _draw_k(rng)
        N = rng.choice((HIDDEN, 3 * HIDDEN, MLP)) if rng.random() < 0.4 else _log_int(rng, 16, MLP)
        M = min(_log_int(rng, 1, 32768), 32768 * HIDDEN * MLP // (K * N))
        return {"kind": kind, "M": M, "K": K, "N": N, "dtype": dtype, "balanced": kind == "layer" and rng.random() < 0.5}
    if kind == "rotary":
        kv_heads = rng.choice((1, 2, 8, 16))
        heads = kv_heads * rng.choice((1, 2, 4))
        head_dim = rng.choice((64, 72, 128))
        T = min(_log_int(rng, 1, 32768), 32768 * 2 * HIDDEN // ((heads + kv_heads) * head_dim))
        rot_dim = rng.choice((head_dim, head_dim, head_dim // 2, 16))
        return {"kind": kind, "T": T, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "rot_dim": rot_dim,
                "interleaved": rng.random() < 0.5, "far": rng.random() < 0.5, "dtype": dtype}
    kv_heads = rng.choice((1, 2, 8))
    heads = kv_heads * rng.choice((1, 2, 4))
    head_dim = rng.choice((64, 72, 80, 96, 128))
    shape = rng.choice(("prompt", "cross", "tokens"))
    sequences = _log_int(rng, 1, 16)
    if shape == "prompt":      # whole prompts, or images and frames
        longest = math.isqrt(150_000_000_000 // (sequences * heads * head_dim))
        queries, keys, causal = min(_log_int(rng, 16, 8192), longest), 0, rng.random() < 0.6
    elif shape == "cross":     # many queries to few keys
        queries = min(_log_int(rng, 64, 16384), 32768 * HIDDEN // (sequences * heads * head_dim))
        keys, causal = _log_int(rng, 8, 300), False
    else:                      # a few new tokens over long keys
        queries, keys, causal = rng.choice((1, 1, 2, 5, 64)), _log_int(rng, 256, 32768), True
    return {"kind": kind, "sequences": sequences, "queries": queries, "keys": keys, "ragged": rng.random() < 0.7,
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "dtype": dtype}


def _lengths(case):
    """Queries and keys of every sequence; the longest is the case's own, the others spread over their logarithm."""
    rng = random.Random(case["sequences"] * 7919 + case["queries"] * 31 + case["keys"])
    top = case["keys"] or case["queries"]
    n = case["sequences"]
    long = [top] + [_log_int(rng, max(1, top // 16), top) if case["ragged"] else top for _ in range(n - 1)]
    rng.shuffle(long)
    return ([case["queries"]] * n, long) if case["keys"] else (long, long)


def work(case):
    kind = case["kind"]
    if kind == "codes":      # (the codes between the two calls are not counted)
        M, K = case["M"], case["K"]
        return {"bytes": 4 * M * K + 4 * K * case["balanced"], "flops": 4 * M * K}
    if kind in ("product", "layer"):
        M, K, N = case["M"], case["K"], case["N"]
        codes = K // 2 + K // 32
        x = M * (codes if kind == "product" else 2 * K) + 4 * K * case["balanced"]
        return {"bytes": x + N * codes + 2 * N + 2 * M * N, "flops": 2 * M * N * K}
    D, H, G = case["head_dim"], case["heads"], case["kv_heads"]
    if kind == "rotary":
        T, R = case["T"], case["rot_dim"]
        return {"bytes": 4 * T * (H + G) * D + 4 * T + 2 * R, "flops": 3 * T * (H + G) * R}
    lq, lk = _lengths(case)
    if case["causal"]:
        pairs = sum(_causal_pairs(a, b) for a, b in zip(lq, lk))
    else:
        pairs = sum(a * b for a, b in zip(lq, lk))
    return {"bytes": 4 * sum(lq) * H * D + 4 * sum(lk) * G * D + 8 * len(lq) + 8, "flops": 4 * pairs * H * D}


def _causal_pairs(q, k):
    """Visible keys over all queries: query i of q sees keys 0 .. i + k - q."""
    first = max(0, q - k)          # queries before this one see none
    n, least = q - first, first + k - q + 1
    return n * least + n * (n - 1) // 2


# ---- inputs ----------------------------------------------------------------------------------------------------

def _activations(g, M, K, dtype):
    """Gaussian bulk, a spread over the channels, a few outlier channels."""
    sigma = torch.exp(torch.rand(K, generator=g, device="cuda") * math.log(100.0) - math.log(10.0))
    sigma = torch.where(torch.rand(K, generator=g, device="cuda") < 0.01, sigma * 50.0, sigma)
    return (torch.randn(M, K, generator=g, device="cuda") * sigma).to(dtype)


def _mask(g, K):
    return torch.exp((torch.rand(K, generator=g, device="cuda") - 0.5) * 2.0 * math.log(4.0))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype, kind = TYPES[case["dtype"]], case["kind"]
    s = {"case": case, "dtype": dtype}
    if kind in ("codes", "layer"):
        s["x"] = _activations(g, case["M"], case["K"], dtype)
        s["chan_mul"] = _mask(g, case["K"]) if case["balanced"] else None
    if kind == "product":
        s["xq"], s["x_scale"] = _pack(_plain_codes(_activations(g, case["M"], case["K"], dtype), None))
    if kind in ("product", "layer"):
        w = torch.randn(case["N"], case["K"], generator=g, device="cuda") * 0.02
        s["wq"], s["w_scale"] = _pack(_plain_codes(w if s.get("chan_mul") is None else w / s["chan_mul"], None))
        s["bias"] = (torch.randn(case["N"], generator=g, device="cuda") * 0.01).to(dtype)
    if kind == "rotary":
        T, H, G, D, R = case["T"], case["heads"], case["kv_heads"], case["head_dim"], case["rot_dim"]
        qkv = torch.randn(T, H + 2 * G, D, generator=g, device="cuda").to(dtype)
        s["q"], s["k"] = qkv[:, :H], qkv[:, H:H + G]          # slices of the QKV layer's output
        if case["far"]:
            s["positions"] = torch.randint(0, 1 << 20, (T,), generator=g, device="cuda", dtype=torch.int32)
        else:
            s["positions"] = torch.arange(T, device="cuda", dtype=torch.int32) % ((T + 1) // 2) + seed % 16
        s["inv_freq"] = (10000.0 ** (torch.arange(R // 2, device="cuda", dtype=torch.float64) * (-2.0 / R))).float()
        s["amplitude"] = 1.2 if case["far"] else 1.0
    if kind == "attention":
        lq, lk = _lengths(case)
        H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
        s["lq"], s["lk"] = lq, lk
        s["cu_q"], s["cu_k"] = (torch.tensor([0] + l, device="cuda").cumsum(0).to(torch.int32) for l in (lq, lk))
        if case["keys"]:
            s["q"] = torch.randn(sum(lq), H, D, generator=g, device="cuda").to(dtype)
            kv = torch.randn(sum(lk), 2 * G, D, generator=g, device="cuda").to(dtype)
            s["k"], s["v"] = kv[:, :G], kv[:, G:]
        else:
            qkv = torch.randn(sum(lq), H + 2 * G, D, generator=g, device="cuda").to(dtype)
            s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------

def _power(e):
    """2^e in fp32, exactly."""
    return ((e + 127) << 23).view(torch.float32)


def _plain_codes(x, chan_mul):
    """(sign and value of every code as fp32 [M,K], exponent of every block's scale [M,K/32])."""
    t = x.float()
    if chan_mul is not None:
        t = t * chan_mul
    b = t.reshape(t.shape[0], -1, 32)
    top = b.abs().amax(-1)
    e = (torch.frexp(top).exponent - 3).clamp(-127, 127)
    e = torch.where(top > 0, e, -127)
    u = b * _power(-e).unsqueeze(-1)
    a = u.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    r = (torch.round(a / step) * step).clamp(max=6.0)
    return torch.copysign(r, u).reshape(t.shape), e


def _pack(codes):
    """Codes in pairs, the even channel in the low half; scales as exponent + 127, rows padded to four."""
    v, e = codes
    a = v.abs()
    n = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (torch.signbit(v).to(torch.uint8) << 3)
    scale = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[1] % 4))
    return n[:, 0::2] | (n[:, 1::2] << 4), scale


def _unpack(q, scale, table):
    K = 2 * q.shape[1]
    n = torch.stack((q & 15, q >> 4), -1).reshape(q.shape[0], K)
    e = scale[:, :K // 32].to(torch.int32) - 127
    return (table[n.long()].reshape(q.shape[0], -1, 32) * _power(e).unsqueeze(-1)).reshape(q.shape[0], K)


def _values(v, e):
    return (v.reshape(*e.shape, 32) * _power(e).unsqueeze(-1)).reshape(v.shape)


def _table(dtype):
    half = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return torch.tensor(half + [-v for v in half], device="cuda", dtype=dtype)


def _plain_product(x, s):
    w = _unpack(s["wq"], s["w_scale"], _table(torch.float32))
    return (x @ w.t() + s["bias"].float()).to(s["dtype"])


def _plain_rotary(x, s):
    R = s["case"]["rot_dim"]
    angle = (s["positions"].double()[:, None] * s["inv_freq"].double()).unsqueeze(1)
    cos, sin = (angle.cos() * s["amplitude"]).float(), (angle.sin() * s["amplitude"]).float()
    t = x[..., :R].float()
    a, b = (t[..., 0::2], t[..., 1::2]) if s["case"]["interleaved"] else (t[..., :R // 2], t[..., R // 2:])
    pair = (a * cos - b * sin, b * cos + a * sin)
    t = torch.stack(pair, -1).flatten(-2) if s["case"]["interleaved"] else torch.cat(pair, -1)
    return torch.cat((t.to(x.dtype), x[..., R:]), -1)


def _plain_sequence(q, k, v, causal):
    """One sequence: q [n,H,D], k and v [m,G,D]."""
    n, H, D = q.shape
    m, G = k.shape[:2]
    q = q.float().transpose(0, 1).reshape(G, -1, D)                                  # a group's heads one after another
    k, v = k.float().transpose(0, 1).contiguous(), v.float().transpose(0, 1).contiguous()
    scores = torch.bmm(q, k.transpose(1, 2).contiguous()).reshape(H, n, m) / math.sqrt(D)
    if causal:
        hidden = torch.arange(m, device=q.device) > torch.arange(n, device=q.device)[:, None] + (m - n)
        scores = scores.masked_fill(hidden, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.bmm(p.reshape(G, -1, m), v).reshape(H, n, D)
    return torch.where(total > 0, out / total, 0.0).transpose(0, 1)


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "codes":
        return _values(*_plain_codes(s["x"], s["chan_mul"])).to(s["dtype"])
    if kind == "product":
        return _plain_product(_unpack(s["xq"], s["x_scale"], _table(torch.float32)), s)
    if kind == "layer":
        return _plain_product(_values(*_plain_codes(s["x"], s["chan_mul"])), s)
    if kind == "rotary":
        return _plain_rotary(s["q"], s), _plain_rotary(s["k"], s)
    parts = zip(s["q"].split(s["lq"]), s["k"].split(s["lk"]), s["v"].split(s["lk"]))
    return torch.cat([_plain_sequence(q, k, v, s["case"]["causal"]).to(s["dtype"]) for q, k, v in parts])


def run(state):
    if not own:
        return _plain(state)
    import paper_2406_02540_amd as vq
    s, kind = state, state["case"]["kind"]
    if kind == "codes":
        return vq.vq_mx4_dequantize(*vq.vq_mx4_quantize(s["x"], s["chan_mul"]), dtype=s["dtype"])
    if kind == "product":
        return vq.vq_gemm_mx4(s["xq"], s["x_scale"], s["wq"], s["w_scale"], s["bias"], dtype=s["dtype"])
    if kind == "layer":
        return vq.vq_linear_mx4(s["x"], s["chan_mul"], s["wq"], s["w_scale"], s["bias"])
    if kind == "rotary":
        return vq.vq_rotary(s["q"], s["k"], s["positions"], s["inv_freq"], interleaved=s["case"]["interleaved"],
                            amplitude=s["amplitude"])
    return vq.vq_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=s["case"]["causal"])


# ---- the definitions in 64 bits --------------------------------------------------------------------------------

def _double_power(e):
    return ((e.clamp(-127, 127) + 1023) << 52).view(torch.float64)


def _exact_codes(x, chan_mul):
    """The values that the codes and scales stand for: the product with the mask is defined as an fp32 number."""
    t = x.double()
    if chan_mul is not None:
        t = (t * chan_mul.double()).float().double()
    t = t.unflatten(1, (-1, 32))
    top = t.abs().max(-1, keepdim=True).values
    scale = _double_power((top.view(torch.int64) >> 52) - 1023 - 2)
    a = (t / scale).abs()
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=x.device, dtype=torch.float64)
    middle = (values[1:] + values[:-1]) / 2
    below, upto = torch.bucketize(a, middle), torch.bucketize(a, middle, right=True)
    n = torch.where((below != upto) & (below % 2 == 0), below, upto)          # a tie: the even code
    return (values[n] * torch.sign(t) * scale).flatten(1)


def _exact_values(q, scale):
    K = 2 * q.shape[1]
    low, high = _table(torch.float64)[(q % 16).long()], _table(torch.float64)[(q // 16).long()]
    v = torch.stack((low, high), 2).reshape(len(q), K // 32, 32)
    return (v * _double_power(scale[:, :K // 32].long() - 127).unsqueeze(2)).reshape(len(q), K)


def _exact_heads(s):
    """Sequence by sequence and head by head."""
    case = s["case"]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    out = torch.zeros_like(q)
    share = case["heads"] // case["kv_heads"]
    at, bt = 0, 0
    for n, m in zip(s["lq"], s["lk"]):
        for h in range(case["heads"]):
            w = q[at:at + n, h] @ k[bt:bt + m, h // share].T * case["head_dim"] ** -0.5
            if case["causal"]:
                w = w.masked_fill(torch.ones_like(w, dtype=torch.bool).triu(m - n + 1), -math.inf)
            out[at:at + n, h] = torch.nan_to_num(torch.softmax(w, 1)) @ v[bt:bt + m, h // share]
        at, bt = at + n, bt + m
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "codes":
        return _exact_codes(s["x"], s["chan_mul"])
    if kind in ("product", "layer"):
        x = _exact_values(s["xq"], s["x_scale"]) if kind == "product" else _exact_codes(s["x"], s["chan_mul"])
        return x @ _exact_values(s["wq"], s["w_scale"]).T + s["bias"].double()
    if kind == "rotary":
        R = case["rot_dim"]
        turn = torch.polar(torch.full((case["T"], R // 2), s["amplitude"], dtype=torch.float64, device="cuda"),
                           torch.outer(s["positions"].double(), s["inv_freq"].double()))[:, None]
        outs = []
        for x in (s["q"], s["k"]):
            y = x.double().clone()
            first, second = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
            z = torch.complex(y[..., first], y[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            outs.append(y)
        return tuple(outs)
    return _exact_heads(s)
