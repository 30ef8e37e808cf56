"""The microscaled format, rotary positions and attention in 64 bits, from their definitions, and the tolerances of the tests.

A rounding to nearest is off by half a step: HALF[t] of the value, and half the smallest subnormal near zero."""
import math

import torch

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF = {t: torch.finfo(t).eps / 2 for t in (F16, BF16, F32)}
TINY = {F16: 2.0 ** -25, BF16: 2.0 ** -134, F32: 2.0 ** -150}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def quantize_mx4(x, chan_mul=None):
    """(magnitude codes with sign [M,K], scale exponents [M,K/32]; -127 where all are zero, 128 where one is not finite), on
    the CPU, by the distance to every number of the format."""
    t = x.detach().cpu().to(torch.float32)
    if chan_mul is not None:
        t = t * chan_mul.detach().cpu()
    t = t.double().reshape(t.shape[0], -1, 32)
    top = t.abs().amax(-1)
    finite = torch.isfinite(t).all(-1)
    exponent = torch.tensor([[math.frexp(v)[1] - 1 if math.isfinite(v) and v > 0 else -1000 for v in row] for row in top.tolist()])
    e = (exponent - 2).clamp(min=-127)
    e = torch.where(finite, e, torch.full_like(e, 128))
    scale = torch.pow(torch.tensor(2.0, dtype=torch.float64), e.double()).unsqueeze(-1)
    u = torch.where(finite.unsqueeze(-1), t / scale, torch.zeros_like(t))
    grid = torch.tensor(E2M1, dtype=torch.float64)
    gap = (u.abs().unsqueeze(-1) - grid).abs()
    best = gap.amin(-1, keepdim=True)
    # the nearest number, of two the one with the even code
    rank = torch.where(gap == best, torch.arange(8) % 2, 9)
    code = rank.argmin(-1)
    sign = torch.where(finite.unsqueeze(-1), torch.signbit(t), torch.zeros_like(t, dtype=torch.bool))
    return (code + 8 * sign).reshape(x.shape), e


def pack_mx4(code, e):
    q = (code[:, 0::2] | (code[:, 1::2] << 4)).to(torch.uint8)
    s = (e + 127).to(torch.uint8)
    return q, torch.nn.functional.pad(s, (0, -s.shape[1] % 4))


def values_mx4(code, e):
    """fp64 values [M,K] (NaN for a block whose scale is)."""
    grid = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float64)
    scale = torch.where(e == 128, torch.nan, torch.pow(torch.tensor(2.0, dtype=torch.float64), e.double()))
    return (grid[code].reshape(code.shape[0], -1, 32) * scale.unsqueeze(-1)).reshape(code.shape)


def unpack_mx4(q, s):
    """Codes and exponents from packed bytes."""
    q, s = q.cpu().long(), s.cpu().long()
    code = torch.stack((q & 15, q >> 4), -1).reshape(q.shape[0], -1)
    return code, s[:, :code.shape[1] // 32] - 127


def product(x, w, bias, dtype):
    """y in 64 bits and what an output may be off: a rounding to dtype, and of the fp32 sums one for each of the 32 values of a
    block and each of the K/32 blocks, at the size that the sum can have on the way."""
    y, size = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        y, size = y + bias.double().cpu(), size + bias.double().cpu().abs()
    return y, HALF[dtype] * y.abs() + TINY[dtype] + (32 + x.shape[1] // 32 + 2) * 2.0 ** -24 * size


def rotary(x, positions, inv_freq, interleaved, amplitude):
    """(rotated in 64 bits, what it may be off): a rounding to x's type, and of the pair's size 2^-21: the angle's own fp32 rounding
    is pi 2^-24, sine and cosine are good to two units of 2^-23, three operations follow."""
    x, p, f = x.double().cpu(), positions.double().cpu(), inv_freq.double().cpu()
    R = 2 * f.shape[0]
    angle = (p[:, None] * f)[:, None, :]
    c, s = angle.cos() * amplitude, angle.sin() * amplitude
    y, size = x.clone(), torch.zeros_like(x)
    ia = torch.arange(R // 2) * 2 if interleaved else torch.arange(R // 2)
    ib = ia + 1 if interleaved else ia + R // 2
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    size[..., ia] = size[..., ib] = (a.abs() + b.abs()) * abs(amplitude)
    return y, size * 2.0 ** -21


def attention(q, k, v, lq, lk, scale, causal, q0=0, k0=0):
    """(out in 64 bits, what it may be off) for the rows of the sequences (0 elsewhere).  Off: a rounding of the output; of the average
    of |v| under the weights a rounding of the weights and twice what a score in fp32 is off (weight and sum); and half of the
    smallest number of the type for every weight, of at least 1 in all."""
    dtype = q.dtype
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    off = torch.zeros_like(out)
    share = q.shape[1] // k.shape[1]
    D = q.shape[2]
    for n, m in zip(lq, lk):
        for h in range(q.shape[1] if n and m else 0):
            Q, K, V = q[q0:q0 + n, h].double(), k[k0:k0 + m, h // share].double(), v[k0:k0 + m, h // share].double()
            s = (Q @ K.t().contiguous()) * scale
            size = (Q.abs() @ K.abs().t().contiguous()) * scale
            if causal:
                hide = torch.arange(m, device=q.device)[None] > torch.arange(n, device=q.device)[:, None] + (m - n)
                s, size = s.masked_fill(hide, -math.inf), size.masked_fill(hide, 0)
            top = s.amax(1, keepdim=True)
            seen = top > -math.inf
            p = torch.exp(s - torch.where(seen, top, 0.0))
            total = p.sum(1, keepdim=True).clamp(min=1e-300)
            p = p / total
            o = p @ V
            score = size.amax(1, keepdim=True) * (D + 4) * 2.0 ** -24
            spread = p @ V.abs()
            # (sums of weights and of products: one rounding a key, the accumulator's way at most m of them)
            rest = (m + 8) * 2.0 ** -24
            t = HALF[dtype] * o.abs() + TINY[dtype] + spread * (HALF[dtype] + 2 * score + rest) + TINY[dtype] * V.abs().sum(0)
            out[q0:q0 + n, h], off[q0:q0 + n, h] = torch.where(seen, o, 0.0), torch.where(seen, t, 0.0)
        q0, k0 = q0 + n, k0 + m
    return out, off


def offsets(lengths, first=0):
    cu = [first]
    for n in lengths:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32)


def check(got, want, off, what=""):
    bad = ~((got.double().cpu() - want.cpu()).abs() <= off.cpu())
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, first at {bad.nonzero()[0].tolist()}: " \
        f"{got.double().cpu()[bad][0].item()} for {want.cpu()[bad][0].item()}, may be off {off.cpu()[bad][0].item()}"
