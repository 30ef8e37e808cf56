"""Attention in a sliding window with first keys that stay visible, against the formula in 64 bits."""
import math
import random

import pytest
import torch

import paper_2406_02540_amd as vq
import more_operator_util as mu
import operator_util as ou
from test_gpu_attention import _data

pytestmark = pytest.mark.gpu
F16, BF16 = ou.F16, ou.BF16


def _run(lq, lk, H, G, D, dtype, left, right, sinks, causal, before=0, behind=0, seed=0, scale=None):
    """Rows in front of and behind the sequences, filled, have to stay."""
    Tq, Tk = before + sum(lq) + behind, sum(lk)
    q, k, v = _data(Tq, Tk, H, G, D, dtype, seed)
    out = torch.full((Tq, H, D), 9.0, dtype=dtype, device="cuda")
    cu_q, cu_k = ou.offsets(lq, before).cuda(), ou.offsets(lk).cuda()
    got = vq.vq_attention_window(q, k, v, cu_q, cu_k, left, right, sinks, softmax_scale=scale, causal=causal, out=out)
    assert got is out
    s = scale if scale is not None else 1 / math.sqrt(D)
    want, off = mu.attention(q, k, v, lq, lk, s, mu.window(left, right, sinks, causal), q0=before)
    end = before + sum(lq)
    ou.check(out[before:end], want[before:end], off[before:end], (lq, lk, H, G, D, left, right, sinks, causal))
    assert (out[:before] == 9).all() and (out[end:] == 9).all()
    again = vq.vq_attention_window(q, k, v, cu_q, cu_k, left, right, sinks, softmax_scale=scale, causal=causal)
    assert torch.equal(out[before:end], again[before:end])


# left, right, sinks, causal
WINDOWS = [(0, 0, 0, True), (0, 0, 0, False), (5, 0, 2, True), (63, 64, 0, False), (100, 7, 70, False), (None, 3, 0, False), (2, None, 1, False),
           (None, None, 0, False), (None, 0, 0, True), (40, None, 500, True), (1, 1, 1, False)]
LENGTHS = [([1], [1]), ([1, 1, 1], [1, 33, 300]), ([3, 0, 2], [5, 7, 0]), ([64, 65, 127, 128, 129], [64, 65, 127, 128, 129]),
           ([5, 200, 1], [700, 3, 1000]), ([300], [1025]), ([513, 7], [63, 1]), ([400], [400])]


@pytest.mark.parametrize("lq,lk", LENGTHS)
@pytest.mark.parametrize("left,right,sinks,causal", WINDOWS)
def test_lengths_and_windows(lq, lk, left, right, sinks, causal):
    _run(lq, lk, 4, 2, 64, F16, left, right, sinks, causal, before=3, behind=5)
    _run(lq, lk, 3, 3, 72, BF16, left, right, sinks, causal)


@pytest.mark.parametrize("D", [8, 24, 40, 64, 72, 80, 88, 96, 104, 128])
@pytest.mark.parametrize("lq,lk", [([270, 30], [270, 130]), ([1, 2], [390, 40])])
def test_head_dims(D, lq, lk):
    _run(lq, lk, 6, 2, D, F16, 50, 0, 3, True)
    _run(lq, lk, 2, 2, D, BF16, 33, 44, 10, False)


@pytest.mark.parametrize("H,G", [(1, 1), (7, 1), (32, 8), (48, 1), (12, 4)])
@pytest.mark.parametrize("lq,lk", [([9, 40], [9, 100]), ([1, 1, 1], [2000, 1, 777]), ([260], [260])])
def test_grouped_heads(H, G, lq, lk):
    _run(lq, lk, H, G, 64, BF16, 20, 0, 1, True)
    _run(lq, lk, H, G, 128, F16, 65, 31, 0, False)


def test_no_limit_is_vq_attention():
    for lq, lk in (([1, 3], [900, 40]), ([200, 77], [200, 300])):
        q, k, v = _data(sum(lq), sum(lk), 4, 2, 128, F16)
        cu_q, cu_k = ou.offsets(lq).cuda(), ou.offsets(lk).cuda()
        for causal in (False, True):
            want = vq.vq_attention(q, k, v, cu_q, cu_k, causal=causal).double()
            got = vq.vq_attention_window(q, k, v, cu_q, cu_k, None, causal=causal).double()
            _, off = mu.attention(q, k, v, lq, lk, 128 ** -0.5, mu.behind(causal))
            assert ((got - want).abs() <= 2 * off).all()


def test_long_keys():
    _run([1, 1, 1], [33000, 517, 20001], 8, 2, 128, F16, 9000, 0, 4, True)
    _run([4], [20000], 8, 8, 72, BF16, 4095, 100, 300, False)
    _run([2, 1, 1], [9000, 0, 31], 4, 1, 64, F16, 5000, None, 0, False)
    _run([130], [9001], 2, 1, 64, BF16, 6000, 0, 65, True)
    _run([2100], [2100], 2, 2, 72, F16, 1024, 1024, 16, False)
    _run([2500, 1700], [2500, 1700], 4, 1, 128, BF16, 511, 0, 4, True)
    _run([1] * 40, [1000 + 77 * i for i in range(40)], 8, 2, 128, BF16, 700, 0, 4, True)


def test_many_short_sequences():
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 20, (2300,), generator=g).tolist()
    _run(lens, lens, 2, 2, 72, F16, 4, 4, 1, False)
    _run(lens, lens[::-1], 2, 1, 64, BF16, 3, 0, 2, True)
    lens = torch.randint(30, 90, (150,), generator=g).tolist()
    _run(lens, lens, 2, 1, 128, F16, 20, 0, 4, True)


def test_a_prompt_among_single_tokens():
    r = random.Random(5)
    lq, lk = [700] + [1] * 60, [900] + [r.randint(1, 2500) for _ in range(60)]
    both = list(zip(lq, lk))
    r.shuffle(both)
    lq, lk = [list(x) for x in zip(*both)]
    _run(lq, lk, 4, 2, 64, F16, 300, 0, 4, True)
    _run(lq, lk, 2, 2, 72, BF16, 128, 64, 0, False)


def test_no_keys_at_all():
    for n in (2, 300):
        q = torch.randn(n, 4, 72, device="cuda").to(F16)
        kv = torch.empty(0, 2, 72, dtype=F16, device="cuda")
        cu = torch.tensor([0, n - 1, n - 1], dtype=torch.int32, device="cuda")
        for args in ((5, 5, 3), (None, None, 0), (0, 0, 70)):
            out = torch.full_like(q, 3.0)
            vq.vq_attention_window(q, kv, kv, cu, torch.zeros(3, dtype=torch.int32, device="cuda"), *args, out=out)
            assert (out[:n - 1] == 0).all() and (out[n - 1] == 3).all()


def test_windows_of_the_largest_numbers():
    top = 2**31 - 1
    for lq, lk in (([300], [300]), ([1, 2], [500, 3]), ([50], [3])):
        for left, right, sinks in ((top, top, 0), (0, top, top), (top, 0, 0), (3, 2, top)):
            for causal in (False, True):
                _run(lq, lk, 2, 1, 64, F16, left, right, sinks, causal)


def test_queries_in_front_of_all_keys():
    # more queries than keys: the first stand in front of key 0 and see what lies to their right, or the first keys
    _run([300], [40], 2, 1, 64, F16, 10, 200, 0, False)
    _run([300], [40], 2, 1, 64, F16, 10, 20, 5, False)
    _run([20, 3], [4, 1], 4, 1, 128, BF16, 10, 6, 1, False)
    _run([300, 150], [40, 149], 2, 1, 72, F16, 10, 0, 5, True)


@pytest.mark.parametrize("n", [1, 300])
def test_scores_that_rise_and_fall(n):
    # large scores first hidden, then seen: the running maximum starts where a row's own window does
    D, m = 72, 900
    g = torch.Generator(device="cuda").manual_seed(4)
    q = (1 + 0.1 * torch.randn(n, 1, D, generator=g, device="cuda")).to(F16)
    for ramp in (torch.linspace(-3, 3, m), torch.linspace(3, -3, m), torch.full((m,), -2.5), (torch.arange(m) % 100).float() * 0.05 - 2):
        k = (torch.randn(m, 1, D, generator=g, device="cuda") * 0.05 + ramp.cuda()[:, None, None]).to(F16)
        v = torch.randn(m, 1, D, generator=g, device="cuda").to(F16)
        cu_q, cu_k = ou.offsets([n]).cuda(), ou.offsets([m]).cuda()
        for left, right, sinks, causal in ((64, 0, 0, True), (64, 0, 3, True), (30, 90, 0, False), (200, 10, 70, False)):
            want, off = mu.attention(q, k, v, [n], [m], 1.0, mu.window(left, right, sinks, causal))
            got = vq.vq_attention_window(q, k, v, cu_q, cu_k, left, right, sinks, softmax_scale=1.0, causal=causal)
            ou.check(got, want, off, (left, right, sinks, causal))


@pytest.mark.parametrize("n,lk", [(1, 3000), (7, 900), (500, 900)])
def test_keys_that_nothing_sees_may_be_anything(n, lk):
    # in front of the window, between the first keys and it, behind the sequence
    left, sinks = 300, 5
    q, k, v = _data(n, lk + 200, 2, 1, 72, F16)
    k, v = k.clone(), v.clone()
    cu_q, cu_k = ou.offsets([n]).cuda(), ou.offsets([lk], 100).cuda()
    for causal, right in ((True, 0), (False, 0)):
        want = vq.vq_attention_window(q, k, v, cu_q, cu_k, left, right, sinks, causal=causal)
        k2, v2 = k.clone(), v.clone()
        first = max(sinks, lk - n - left)
        for t, bad in ((k2, float("nan")), (v2, float("inf")), (v2, float("nan"))):
            t[:100] = bad
            t[100 + lk:] = bad
            t[100 + sinks:100 + first] = bad
        got = vq.vq_attention_window(q, k2, v2, cu_q, cu_k, left, right, sinks, causal=causal)
        assert torch.equal(got, want) and not got.isnan().any()


def test_hidden_keys_that_are_not_finite():
    n = 600
    q, k, v = _data(n, n, 2, 2, 64, BF16)
    k = k.clone()
    cu = ou.offsets([n]).cuda()
    want = vq.vq_attention_window(q, k, v, cu, cu, 50, 0, 2, causal=True)
    k[300:310] = float("nan")
    got = vq.vq_attention_window(q, k, v, cu, cu, 50, 0, 2, causal=True)
    hit = torch.zeros(n, dtype=torch.bool)
    hit[300:360] = True
    assert torch.equal(got[~hit], want[~hit]) and got[hit].isnan().all()
    # and values, in blocks of 128 rows none of which sees them
    v = v.clone()
    v[300] = float("inf")
    k = _data(n, n, 2, 2, 64, BF16)[1]
    got = vq.vq_attention_window(q, k, v, cu, cu, 50, 0, 2, causal=True)
    assert torch.equal(got[:256], want[:256]) and torch.equal(got[384:], want[384:])


@pytest.mark.parametrize("n,m", [(1, 600), (200, 200)])
def test_views(n, m):
    H, G, D = 4, 2, 72
    qkv = torch.randn(max(n, m), H + 2 * G, D, generator=torch.Generator().manual_seed(1)).to(F16).cuda()
    q, k, v = qkv[:n, :H], qkv[:m, H:H + G], qkv[:m, H + G:]
    cu_q, cu_k = ou.offsets([n]).cuda(), ou.offsets([m]).cuda()
    seen = mu.window(70, 0, 3, True)
    want, off = mu.attention(q, k, v, [n], [m], D ** -0.5, seen)
    ou.check(vq.vq_attention_window(q, k, v, cu_q, cu_k, 70, 0, 3, causal=True), want, off, "slices")
    major = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    big = torch.full((n, H + 1, D + 8), 5.0, dtype=F16, device="cuda")
    vq.vq_attention_window(*major, cu_q, cu_k, 70, 0, 3, causal=True, out=big[:, :H, :D])
    ou.check(big[:, :H, :D], want, off, "head-major")
    assert (big[:, H] == 5).all() and (big[..., D:] == 5).all()
    k1, v1 = (t[:, :1].expand(m, G, D) for t in (k, v))
    want, off = mu.attention(q, k1, v1, [n], [m], D ** -0.5, seen)
    ou.check(vq.vq_attention_window(q, k1, v1, cu_q, cu_k, 70, 0, 3, causal=True), want, off, "shared")


def test_offsets_beyond_32_bits():
    # keys 4 MiB apart: the window lies 5 GiB into the buffer
    m, D = 1300, 64
    buf = torch.zeros(m, 1 << 21, dtype=F16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    buf[:, :2 * D] = torch.randn(m, 2 * D, generator=g, device="cuda").to(F16)
    k, v = buf[:, None, :D], buf[:, None, D:2 * D]
    for n in (1, 100):
        q = torch.randn(n, 1, D, generator=g, device="cuda").to(F16)
        want, off = mu.attention(q, k, v, [n], [m], D ** -0.5, mu.window(200, 0, 4, True))
        got = vq.vq_attention_window(q, k, v, ou.offsets([n]).cuda(), ou.offsets([m]).cuda(), 200, 0, 4, causal=True)
        ou.check(got, want, off, n)


@pytest.mark.parametrize("H,G,Tk", [(2, 1, 90), (1, 1, 4000), (6, 2, 4000)])
def test_offsets_outside_the_tensors(H, G, Tk):
    Tq, D = 100, 64
    for cu_q, cu_k in (([-20, 40, 100000, 300, 120], [-7, 30, 200000, 95, 1 << 30]), ([0, 40, 20, -5, -7], [0, 30, 10, -4, -9])):
        room = torch.full((Tq + 64, H, D), 5.0, dtype=F16, device="cuda")
        q, k, v = _data(Tq, Tk, H, G, D, F16)
        cu = [torch.tensor(c, dtype=torch.int32).cuda() for c in (cu_q, cu_k)]
        vq.vq_attention_window(q, k, v, *cu, 1000, 0, 3, causal=True, out=room[32:32 + Tq])
        torch.cuda.synchronize()
        assert (room[:32] == 5).all() and (room[32 + Tq:] == 5).all()


@pytest.mark.parametrize("lq,lk", [([1, 1], [4000, 900]), ([150, 90], [150, 90])])
def test_captured_and_replayed(lq, lk):
    H, G, D = 8, 2, 128
    args = (700, 0, 4)
    sets = [_data(sum(lq), sum(lk), H, G, D, F16, seed) for seed in range(3)]
    q, k, v = (t.clone() for t in sets[0])
    cu_q, cu_k = ou.offsets(lq).cuda(), ou.offsets(lk).cuda()
    bytes_ = vq.vq_attention_window_workspace_bytes(len(lq), sum(lq), sum(lk), H, G, D, True, *args)
    work = torch.empty(max(bytes_, 16), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    vq.vq_attention_window(q, k, v, cu_q, cu_k, *args, causal=True, out=out, workspace=work)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vq.vq_attention_window(q, k, v, cu_q, cu_k, *args, causal=True, out=out, workspace=work)
    for s in (2, 0, 1):
        for a, b in zip((q, k, v), sets[s]):
            a.copy_(b)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, vq.vq_attention_window(*sets[s], cu_q, cu_k, *args, causal=True))


def test_two_streams_at_once():
    lq, lk = [1] * 8, [3000] * 8
    q, k, v = _data(8, 24000, 8, 2, 128, F16)
    cu_q, cu_k = ou.offsets(lq).cuda(), ou.offsets(lk).cuda()
    want = vq.vq_attention_window(q, k, v, cu_q, cu_k, 2000, 0, 4, causal=True)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [vq.vq_attention_window(q, k, v, cu_q, cu_k, 2000, 0, 4, causal=True, stream=s) for _ in range(5) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("T", [300, 5])
def test_block(T):
    """QKV layer, norm and positions in place, attention in a window on the slices, output layer: each step against its definition on what
    the step before gave."""
    hidden, H, D, sections = 1152, 16, 72, (8, 14, 14)
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, hidden, generator=g).to(F16)
    cm = torch.exp(torch.randn(hidden, generator=g) * 0.3)
    w1, w2 = torch.randn(3 * hidden, hidden, generator=g) * 0.03, torch.randn(hidden, hidden, generator=g) * 0.03
    b1 = (torch.randn(3 * hidden, generator=g) * 0.1).to(F16)
    q1, s1 = vq.vq_mx4_quantize(w1.cuda(), (1 / cm).cuda())
    q2, s2 = vq.vq_mx4_quantize(w2.cuda())
    lens = [T - 2, 2]
    at = torch.arange(T)
    p = torch.stack((at // 60, at % 60 // 10, at % 10)).to(torch.int32).cuda()
    f = torch.cat([vq.vq_rotary_frequencies(2 * n)[0] for n in sections]).cuda()
    nw = [(1 + 0.2 * torch.randn(D, generator=g)).cuda() for _ in range(2)]
    cu = ou.offsets(lens).cuda()

    qkv = vq.vq_linear_mx4(x.cuda(), cm.cuda(), q1, s1, b1.cuda())
    want, off = ou.product(ou.values_mx4(*ou.quantize_mx4(x, cm)), ou.values_mx4(*ou.unpack_mx4(q1, s1)), b1, F16)
    ou.check(qkv, want, off, "qkv")
    heads = qkv.view(T, 3 * H, D)
    q, k, v = heads[:, :H], heads[:, H:2 * H], heads[:, 2 * H:]
    wants = [mu.turn(*mu.norm(t, w, None, "rms", 1e-6), p, f, sections, "neighbours", 1.0) for t, w in zip((q, k), nw)]
    vq.vq_norm_rotary(q, k, *nw, positions=p, inv_freq=f, sections=sections, pairing="neighbours", q_out=q, k_out=k)
    for name, t, (want, off) in zip("qk", (q, k), wants):
        ou.check(t, want, mu.rounded(want, off, F16), name)
    o = vq.vq_attention_window(q, k, v, cu, cu, 100, 50, sinks=4)
    want, off = mu.attention(q, k, v, lens, lens, D ** -0.5, mu.window(100, 50, 4, False))
    ou.check(o, want, off, "attention")
    y = vq.vq_linear_mx4(o.view(T, hidden), None, q2, s2)
    want, off = ou.product(ou.values_mx4(*ou.quantize_mx4(o.view(T, hidden))), ou.values_mx4(*ou.unpack_mx4(q2, s2)), None, F16)
    ou.check(y, want, off, "output layer")
