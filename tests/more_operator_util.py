"""Rotary positions of several axes, norms of heads, attention in a window and behind a prefix in 64 bits, from their definitions, and the
tolerances of their tests (roundings as in operator_util)."""
import math

import torch

from operator_util import HALF, TINY

U = 2.0 ** -24        # half a step of fp32


def channels_of(sections, pairing):
    """[(axis, number of the pair, first channel, second channel)]."""
    out, n, f = [], sum(sections), 0
    for axis, size in enumerate(sections):
        for i in range(size):
            pair = f + i
            out.append((axis, pair, *{"halves": (pair, pair + n), "neighbours": (2 * pair, 2 * pair + 1),
                                      "axis_halves": (2 * f + i, 2 * f + i + size)}[pairing]))
        f += size
    return out


def turn(x, off, positions, inv_freq, sections, pairing, amplitude):
    """x [T,H,D] in 64 bits, off by up to `off`: (turned, what it may be off before its last rounding).  Of the pair's size 2^-21: the angle's
    own fp32 rounding is pi 2^-24, sine and cosine are good to two units of 2^-23, three operations follow."""
    pairs = channels_of(sections, pairing)
    axis, pair, first, second = (torch.tensor(c) for c in zip(*pairs))
    p, f = positions.double().cpu(), inv_freq.double().cpu()
    angle = (p[axis].t() * f[pair])[:, None, :]
    c, s = angle.cos() * amplitude, angle.sin() * amplitude
    y, o = x.clone(), off.clone()
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    both = (off[..., first] + off[..., second]) * abs(amplitude) * 1.001 + (a.abs() + b.abs()) * abs(amplitude) * 2.0 ** -21
    o[..., first] = o[..., second] = both
    return y, o


def norm(x, weight, bias, kind, eps):
    """(normed in 64 bits, what an fp32 evaluation may be off).  A sum of D values in any order is off by D U of the sum of their sizes; half of
    that for a root; five operations more.  Mean and variance: the mean's error moves every difference, and the variance by at most twice it
    times the mean size of the differences, which the root of the variance exceeds."""
    x = x.double().cpu()
    D = x.shape[-1]
    moved = torch.zeros_like(x[..., :1])
    if kind == "layer":
        moved = (D + 2) * U * x.abs().mean(-1, keepdim=True)
        x = x - x.mean(-1, keepdim=True)
    size = torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    w = torch.ones(D, dtype=torch.float64) if weight is None else weight.double().cpu()
    b = torch.zeros(D, dtype=torch.float64) if bias is None else bias.double().cpu()
    y = x / size * w
    off = moved / size * w.abs() * 1.001 + y.abs() * ((D / 2 + 8) * U + 1.001 * moved / size)
    return y + b, off + (y + b).abs() * U


def rounded(want, off, dtype):
    return off + HALF[dtype] * (want.abs() + off) + TINY[dtype]


def window(left, right, sinks, causal):
    """seen(n, m): bool [n, m]."""
    def seen(n, m):
        p = torch.arange(n)[:, None] + (m - n)
        j = torch.arange(m)[None]
        s = torch.ones(n, m, dtype=torch.bool)
        if left is not None and left >= 0:
            s &= j >= p - left
        if right is not None and right >= 0 and not causal:
            s &= j <= p + right
        s |= j < sinks
        return s & (j <= p) if causal else s
    return seen


def behind(causal):
    def seen(n, m):
        s = torch.ones(n, m, dtype=torch.bool)
        return s & (torch.arange(m)[None] <= torch.arange(n)[:, None] + (m - n)) if causal else s
    return seen


def attention(q, k, v, lq, lk, scale, seen, q0=0, k0=0, prefix_k=None, prefix_v=None):
    """(out in 64 bits, what it may be off) for the rows of the sequences (0 elsewhere); a query sees the prefix and the keys that
    seen(n, m) gives.  Off: as operator_util.attention."""
    dtype = q.dtype
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    off = torch.zeros_like(out)
    share, D = q.shape[1] // k.shape[1], q.shape[2]
    for n, m in zip(lq, lk):
        hide = ~seen(n, m).to(q.device)
        for h in range(q.shape[1] if n else 0):
            Q, K, V = q[q0:q0 + n, h].double(), k[k0:k0 + m, h // share].double(), v[k0:k0 + m, h // share].double()
            hidden = hide
            if prefix_k is not None:
                P = prefix_k.shape[0]
                K, V = torch.cat((prefix_k[:, h // share].double(), K)), torch.cat((prefix_v[:, h // share].double(), V))
                hidden = torch.cat((torch.zeros(n, P, dtype=torch.bool, device=q.device), hide), 1)
            if K.shape[0] == 0:
                continue
            s = ((Q @ K.t().contiguous()) * scale).masked_fill(hidden, -math.inf)
            size = ((Q.abs() @ K.abs().t().contiguous()) * scale).masked_fill(hidden, 0)
            top = s.amax(1, keepdim=True)
            any_ = top > -math.inf
            p = torch.exp(s - torch.where(any_, top, 0.0))
            p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
            V = torch.where((~hidden).any(0)[:, None], V, 0.0)
            o = p @ V
            score = size.amax(1, keepdim=True) * (D + 4) * U
            rest = (K.shape[0] + 8) * U
            t = HALF[dtype] * o.abs() + TINY[dtype] + (p @ V.abs()) * (HALF[dtype] + 2 * score + rest) + TINY[dtype] * V.abs().sum(0)
            out[q0:q0 + n, h], off[q0:q0 + n, h] = torch.where(any_, o, 0.0), torch.where(any_, t, 0.0)
        q0, k0 = q0 + n, k0 + m
    return out, off
