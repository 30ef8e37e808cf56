"""Attention of sequences behind keys that all of them share, against the formula in 64 bits."""
import math

import pytest
import torch

import paper_2406_02540_amd as vq
import more_operator_util as mu
import operator_util as ou
from test_gpu_attention import _data

pytestmark = pytest.mark.gpu
F16, BF16 = ou.F16, ou.BF16


def _prefix(P, G, D, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 31 + P + D)
    kv = torch.randn(P, 2 * G + 1, D, generator=g, device="cuda").to(dtype)      # (other strides than k's and v's)
    return kv[:, :G], kv[:, G:2 * G]


def _run(lq, lk, P, H, G, D, dtype, causal, before=0, behind=0, seed=0, scale=None):
    """Rows in front of and behind the sequences, filled, have to stay."""
    Tq, Tk = before + sum(lq) + behind, sum(lk)
    q, k, v = _data(Tq, Tk, H, G, D, dtype, seed)
    pk, pv = _prefix(P, G, D, dtype, seed)
    out = torch.full((Tq, H, D), 9.0, dtype=dtype, device="cuda")
    cu_q, cu_k = ou.offsets(lq, before).cuda(), ou.offsets(lk).cuda()
    got = vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k, softmax_scale=scale, causal=causal, out=out)
    assert got is out
    s = scale if scale is not None else 1 / math.sqrt(D)
    want, off = mu.attention(q, k, v, lq, lk, s, mu.behind(causal), before, 0, pk, pv)
    end = before + sum(lq)
    ou.check(out[before:end], want[before:end], off[before:end], (lq, lk, P, H, G, D, causal))
    assert (out[:before] == 9).all() and (out[end:] == 9).all()
    again = vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k, softmax_scale=scale, causal=causal)
    assert torch.equal(out[before:end], again[before:end])


LENGTHS = [([1], [1]), ([1, 1, 1], [1, 33, 300]), ([3, 0, 2], [5, 7, 0]), ([64, 65, 127, 128, 129], [64, 65, 127, 128, 129]),
           ([5, 200, 1], [700, 3, 1000]), ([300], [1025]), ([513, 7], [63, 1]), ([400, 90], [400, 90]), ([1] * 40, [7] * 40)]


@pytest.mark.parametrize("lq,lk", LENGTHS)
@pytest.mark.parametrize("P", [0, 1, 63, 64, 200, 1500])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(lq, lk, P, causal):
    _run(lq, lk, P, 4, 2, 64, F16, causal, before=3, behind=5)
    _run(lq, lk, P, 3, 3, 72, BF16, causal)


@pytest.mark.parametrize("D", [8, 24, 40, 64, 72, 80, 88, 96, 104, 128])
@pytest.mark.parametrize("lq,lk", [([270, 30], [270, 130]), ([1, 2], [390, 40])])
def test_head_dims(D, lq, lk):
    _run(lq, lk, 333, 6, 2, D, F16, True)
    _run(lq, lk, 70, 2, 2, D, BF16, False)


@pytest.mark.parametrize("H,G", [(1, 1), (7, 1), (32, 8), (48, 1), (12, 4)])
@pytest.mark.parametrize("lq,lk", [([9, 40], [9, 100]), ([1, 1, 1], [2000, 1, 777]), ([260], [260]), ([1] * 70, [20] * 70)])
def test_grouped_heads(H, G, lq, lk):
    _run(lq, lk, 500, H, G, 64, BF16, True)
    _run(lq, lk, 129, H, G, 128, F16, False)


def test_long_prefixes():
    _run([1, 1, 1], [30, 517, 1], 33000, 8, 2, 128, F16, True)
    _run([1] * 64, [40 + i for i in range(64)], 8192, 8, 2, 128, BF16, True)
    _run([7] * 5, [301, 7, 20, 100, 31], 30011, 16, 2, 64, F16, True)
    _run([2, 1, 1], [9000, 0, 31], 5000, 4, 1, 64, F16, False)
    _run([130], [131], 9001, 2, 1, 64, BF16, True)
    _run([1000, 700], [1000, 700], 300, 2, 2, 72, F16, False)
    _run([16] * 9, [16] * 9, 2777, 4, 4, 80, BF16, True)


def test_many_short_sequences():
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 20, (2300,), generator=g).tolist()
    _run(lens, lens, 100, 2, 2, 72, F16, False)
    _run(lens, lens[::-1], 65, 2, 1, 64, BF16, True)
    lens = torch.randint(30, 90, (150,), generator=g).tolist()
    _run(lens, lens, 400, 2, 1, 128, F16, True)


def test_a_prompt_among_single_tokens():
    _run([700] + [1] * 60, [900] + [1 + 40 * i for i in range(60)], 1000, 4, 2, 64, F16, True)
    _run([1] * 30 + [333] + [1] * 30, [5] * 61, 77, 2, 2, 72, BF16, False)


def test_blocks_of_rows_that_begin_in_the_prefix_and_behind_it():
    # one sequence of several blocks of rows among single tokens, its keys divided: later blocks see more keys, so that a workgroup's part begins in
    # the prefix for one block and behind it for the next, and k, v lie otherwise than the prefix
    for lq, lk in (([1000] + [1] * 32, [1000] + [9] * 32), ([1] * 33 + [1020], [3] * 33 + [1100])):
        _run(lq, lk, 600, 1, 1, 64, F16, True)
        _run(lq, lk, 600, 1, 1, 72, BF16, True, before=1, behind=2)


def test_no_own_keys_and_no_prefix():
    for n in (2, 300):
        q = torch.randn(n, 4, 72, device="cuda").to(F16)
        none = torch.empty(0, 2, 72, dtype=F16, device="cuda")
        cu, zeros = torch.tensor([0, n - 1, n - 1], dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 3.0)
        vq.vq_attention_prefix(q, none, none, none, none, cu, zeros, out=out)
        assert (out[:n - 1] == 0).all() and (out[n - 1] == 3).all()
        pk, pv = _prefix(50, 2, 72, F16)
        vq.vq_attention_prefix(q, pk, pv, none, none, cu, zeros, out=out, causal=True)
        want, off = mu.attention(q, none, none, [n - 1], [0], 72 ** -0.5, mu.behind(True), 0, 0, pk, pv)
        ou.check(out[:n - 1], want[:n - 1], off[:n - 1])
        assert (out[n - 1] == 3).all()


def test_prefix_as_a_part_of_every_sequence():
    # what vq_attention gives with the shared keys in front of each sequence's own
    lq, lk, P = [1, 5, 2], [9, 70, 2], 300
    q, k, v = _data(sum(lq), sum(lk), 4, 2, 128, F16)
    pk, pv = _prefix(P, 2, 128, F16)
    got = vq.vq_attention_prefix(q, pk, pv, k, v, ou.offsets(lq).cuda(), ou.offsets(lk).cuda(), causal=True).double()
    ks, vs = (torch.cat([t for part in x.split(lk) for t in (p, part)]) for x, p in ((k, pk), (v, pv)))
    longer = [P + m for m in lk]
    want = vq.vq_attention(q, ks, vs, ou.offsets(lq).cuda(), ou.offsets(longer).cuda(), causal=True).double()
    _, off = ou.attention(q, ks, vs, lq, longer, 128 ** -0.5, True)
    assert ((got - want).abs() <= 2 * off).all()


@pytest.mark.parametrize("n", [1, 300])
def test_scores_far_apart(n):
    # the prefix's scores far above, far below, and of the size of the own keys'
    D, m, P = 72, 200, 400
    g = torch.Generator(device="cuda").manual_seed(4)
    q = (1 + 0.1 * torch.randn(n, 1, D, generator=g, device="cuda")).to(F16)
    for a, b in ((-3, 3), (3, -3), (-2.5, -2.5), (0, 1)):
        k, pk = ((torch.randn(x, 1, D, generator=g, device="cuda") * 0.05 + c).to(F16) for x, c in ((m, a), (P, b)))
        v, pv = (torch.randn(x, 1, D, generator=g, device="cuda").to(F16) for x in (m, P))
        want, off = mu.attention(q, k, v, [n], [m], 1.0, mu.behind(True), 0, 0, pk, pv)
        got = vq.vq_attention_prefix(q, pk, pv, k, v, ou.offsets([n]).cuda(), ou.offsets([m]).cuda(), softmax_scale=1.0, causal=True)
        ou.check(got, want, off, (a, b))


@pytest.mark.parametrize("n", [1, 150])
def test_keys_behind_a_sequence_do_not_matter(n):
    q, k, v = _data(2 * n, 400, 2, 1, 72, F16)
    k, v = k.clone(), v.clone()
    P = 130
    room = torch.randn(P + 60, 2, 72, device="cuda").to(F16)
    pk, pv = room[30:30 + P, :1], room[30:30 + P, 1:]
    cu_q, cu_k = ou.offsets([n, n]).cuda(), ou.offsets([150, 41], 100).cuda()
    want = vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k)
    k[:100] = k[291:] = float("nan")
    v[:100] = v[291:] = float("inf")
    room[:30] = room[30 + P:] = float("nan")
    got = vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k)
    assert torch.equal(got, want) and not got.isnan().any()


@pytest.mark.parametrize("n,m", [(1, 600), (200, 200)])
def test_views(n, m):
    H, G, D, P = 4, 2, 72, 90
    qkv = torch.randn(max(n, m), H + 2 * G, D, generator=torch.Generator().manual_seed(1)).to(F16).cuda()
    q, k, v = qkv[:n, :H], qkv[:m, H:H + G], qkv[:m, H + G:]
    pk, pv = _prefix(P, G, D, F16)
    cu_q, cu_k = ou.offsets([n]).cuda(), ou.offsets([m]).cuda()
    want, off = mu.attention(q, k, v, [n], [m], D ** -0.5, mu.behind(True), 0, 0, pk, pv)
    ou.check(vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k, causal=True), want, off, "slices")
    qm, pkm, pvm, km, vm = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, pk, pv, k, v))
    big = torch.full((n, H + 1, D + 8), 5.0, dtype=F16, device="cuda")
    vq.vq_attention_prefix(qm, pkm, pvm, km, vm, cu_q, cu_k, causal=True, out=big[:, :H, :D])
    ou.check(big[:, :H, :D], want, off, "head-major")
    assert (big[:, H] == 5).all() and (big[..., D:] == 5).all()
    one = [t[:, :1].expand(t.shape[0], G, D) for t in (pk, pv, k, v)]
    want, off = mu.attention(q, one[2], one[3], [n], [m], D ** -0.5, mu.behind(False), 0, 0, one[0], one[1])
    ou.check(vq.vq_attention_prefix(q, *one, cu_q, cu_k), want, off, "shared")


def test_offsets_beyond_32_bits():
    # keys of the prefix 4 MiB apart: the last ones lie 5 GiB into the buffer
    P, D = 1300, 64
    buf = torch.zeros(P, 1 << 21, dtype=F16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    buf[:, :2 * D] = torch.randn(P, 2 * D, generator=g, device="cuda").to(F16)
    pk, pv = buf[:, None, :D], buf[:, None, D:2 * D]
    for lq, lk in (([1, 2], [5, 9]), ([100], [60])):
        q, k, v = _data(sum(lq), sum(lk), 1, 1, D, F16)
        want, off = mu.attention(q, k, v, lq, lk, D ** -0.5, mu.behind(True), 0, 0, pk, pv)
        got = vq.vq_attention_prefix(q, pk, pv, k, v, ou.offsets(lq).cuda(), ou.offsets(lk).cuda(), causal=True)
        ou.check(got, want, off, lq)


@pytest.mark.parametrize("H,G,Tk,P", [(2, 1, 90, 40), (1, 1, 4000, 9000), (6, 2, 4000, 700)])
def test_offsets_outside_the_tensors(H, G, Tk, P):
    Tq, D = 100, 64
    for cu_q, cu_k in (([-20, 40, 100000, 300, 120], [-7, 30, 200000, 95, 1 << 30]), ([0, 40, 20, -5, -7], [0, 30, 10, -4, -9])):
        room = torch.full((Tq + 64, H, D), 5.0, dtype=F16, device="cuda")
        q, k, v = _data(Tq, Tk, H, G, D, F16)
        cu = [torch.tensor(c, dtype=torch.int32).cuda() for c in (cu_q, cu_k)]
        vq.vq_attention_prefix(q, *_prefix(P, G, D, F16), k, v, *cu, causal=True, out=room[32:32 + Tq])
        torch.cuda.synchronize()
        assert (room[:32] == 5).all() and (room[32 + Tq:] == 5).all()


@pytest.mark.parametrize("lq,lk,P", [([1, 1], [400, 900], 5000), ([1] * 50, [20] * 50, 3000), ([150, 90], [150, 90], 200)])
def test_captured_and_replayed(lq, lk, P):
    H, G, D = 8, 2, 128
    sets = [(*_data(sum(lq), sum(lk), H, G, D, F16, seed), *_prefix(P, G, D, F16, seed)) for seed in range(3)]
    q, k, v, pk, pv = (t.clone() for t in sets[0])
    cu_q, cu_k = ou.offsets(lq).cuda(), ou.offsets(lk).cuda()
    bytes_ = vq.vq_attention_prefix_workspace_bytes(len(lq), sum(lq), P, sum(lk), H, G, D)
    work = torch.empty(max(bytes_, 16), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k, causal=True, out=out, workspace=work)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k, causal=True, out=out, workspace=work)
    for s in (2, 0, 1):
        for a, b in zip((q, k, v, pk, pv), sets[s]):
            a.copy_(b)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        sq, sk, sv, spk, spv = sets[s]
        assert torch.equal(out, vq.vq_attention_prefix(sq, spk, spv, sk, sv, cu_q, cu_k, causal=True))


def test_two_streams_at_once():
    lq, lk, P = [1] * 8, [300] * 8, 6000
    q, k, v = _data(8, 2400, 8, 2, 128, F16)
    pk, pv = _prefix(P, 2, 128, F16)
    cu_q, cu_k = ou.offsets(lq).cuda(), ou.offsets(lk).cuda()
    want = vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k, causal=True)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k, causal=True, stream=s) for _ in range(5) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_images_of_one_caption():
    """Keys and values of a caption by its own layer, norm and positions of the images' slices, attention behind the caption: each step against
    its definition on what the step before gave."""
    H, D, P, n, images, sections = 16, 72, 120, 100, 3, (18, 18)
    g = torch.Generator().manual_seed(11)
    text = torch.randn(P, 512, generator=g).to(F16)
    w = torch.randn(2 * H * D, 512, generator=g) * 0.05
    wq, ws = vq.vq_mx4_quantize(w.cuda())
    kv = vq.vq_linear_mx4(text.cuda(), None, wq, ws).view(P, 2 * H, D)
    want, off = ou.product(ou.values_mx4(*ou.quantize_mx4(text)), ou.values_mx4(*ou.unpack_mx4(wq, ws)), None, F16)
    ou.check(kv.reshape(P, -1), want, off, "caption")
    qkv = torch.randn(images * n, 3 * H, D, generator=g).to(F16).cuda()
    q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
    at = torch.arange(n).repeat(images)
    p = torch.stack((at // 10, at % 10)).to(torch.int32).cuda()
    f = torch.cat([vq.vq_rotary_frequencies(2 * s)[0] for s in sections]).cuda()
    wants = [mu.turn(*mu.norm(t, None, None, "layer", 1e-6), p, f, sections, "axis_halves", 1.0) for t in (q, k)]
    vq.vq_norm_rotary(q, k, norm="layer", positions=p, inv_freq=f, sections=sections, pairing="axis_halves", q_out=q, k_out=k)
    for name, t, (want, off) in zip("qk", (q, k), wants):
        ou.check(t, want, mu.rounded(want, off, F16), name)
    cu = ou.offsets([n] * images).cuda()
    o = vq.vq_attention_prefix(q, kv[:, :H], kv[:, H:], k, v, cu, cu)
    want, off = mu.attention(q, k, v, [n] * images, [n] * images, D ** -0.5, mu.behind(False), 0, 0, kv[:, :H], kv[:, H:])
    ou.check(o, want, off, "attention")
