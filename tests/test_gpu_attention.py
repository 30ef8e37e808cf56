"""Attention over packed sequences against the formula in 64 bits."""
import math

import pytest
import torch

import paper_2406_02540_amd as vq
import operator_util as ou

pytestmark = pytest.mark.gpu
F16, BF16 = ou.F16, ou.BF16


def _data(Tq, Tk, H, G, D, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 77 + Tq + 3 * Tk + D)
    q = torch.randn(Tq, H, D, generator=g, device="cuda").to(dtype)
    kv = torch.randn(Tk, 2 * G, D, generator=g, device="cuda").to(dtype)
    return q, kv[:, :G], kv[:, G:]


def _run(lq, lk, H, G, D, dtype, causal, scale=None, before=0, behind=0, seed=0):
    """Rows in front of and behind the sequences, filled, have to stay."""
    Tq, Tk = before + sum(lq) + behind, sum(lk)
    q, k, v = _data(Tq, Tk, H, G, D, dtype, seed)
    out = torch.full((Tq, H, D), 9.0, dtype=dtype, device="cuda")
    cu_q, cu_k = ou.offsets(lq, before).cuda(), ou.offsets(lk).cuda()
    got = vq.vq_attention(q, k, v, cu_q, cu_k, softmax_scale=scale, causal=causal, out=out)
    assert got is out
    s = scale if scale is not None else 1 / math.sqrt(D)
    want, off = ou.attention(q, k, v, lq, lk, s, causal, q0=before)
    end = before + sum(lq)
    ou.check(out[before:end], want[before:end], off[before:end], (lq, lk, H, G, D, causal))
    assert (out[:before] == 9).all() and (out[end:] == 9).all()
    assert torch.equal(out[before:end], vq.vq_attention(q, k, v, cu_q, cu_k, softmax_scale=scale, causal=causal)[before:end])


CASES = [
    # lengths of queries, of keys
    ([1], [1]),
    ([1, 1, 1], [1, 33, 300]),
    ([3, 0, 2], [5, 7, 0]),
    ([32, 31, 33], [32, 31, 33]),
    ([64, 65, 127, 128, 129], [64, 65, 127, 128, 129]),
    ([100, 1], [37, 500]),
    ([5, 200, 1], [700, 3, 1000]),
    ([300], [1025]),
    ([513, 7], [63, 1]),
]


@pytest.mark.parametrize("lq,lk", CASES)
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(lq, lk, D, causal):
    _run(lq, lk, 4, 2, D, F16, causal, before=3, behind=5)
    _run(lq, lk, 3, 3, D, BF16, causal)


@pytest.mark.parametrize("D", [8, 16, 24, 40, 56, 80, 88, 96, 104, 112, 120])
@pytest.mark.parametrize("lq,lk", [([70, 30], [70, 130]), ([1, 1], [90, 40])])
def test_head_dims(D, lq, lk):
    _run(lq, lk, 6, 2, D, F16, True)
    _run(lq, lk, 2, 2, D, BF16, False)


@pytest.mark.parametrize("H,G", [(1, 1), (7, 1), (32, 8), (48, 1), (12, 4)])
@pytest.mark.parametrize("lq,lk", [([9, 40], [9, 100]), ([1, 1, 1], [2000, 1, 777]), ([260], [260])])
def test_grouped_heads(H, G, lq, lk):
    _run(lq, lk, H, G, 64, BF16, True)
    _run(lq, lk, H, G, 128, F16, False)


def test_long_keys_in_parts():
    _run([1, 1], [33000, 517], 8, 2, 128, F16, True)
    _run([4], [20000], 8, 8, 72, BF16, False)
    _run([2, 1, 1], [9000, 0, 31], 4, 1, 64, F16, True)
    _run([40], [16000], 4, 4, 128, F16, True)
    _run([130], [9001], 2, 1, 64, BF16, False)


def test_many_short_sequences():
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 20, (700,), generator=g).tolist()
    _run(lens, lens, 2, 2, 72, F16, False)
    _run(lens, lens[::-1], 2, 1, 64, BF16, True)
    lens = torch.randint(30, 90, (150,), generator=g).tolist()
    _run(lens, lens, 2, 1, 128, F16, True)


def test_long_prompt():
    _run([2500, 1700], [2500, 1700], 2, 1, 128, BF16, True)
    _run([3001], [3001], 2, 2, 72, F16, False)


def test_no_keys_at_all():
    for n in (2, 300):
        q = torch.randn(n, 4, 72, device="cuda").to(F16)
        kv = torch.empty(0, 2, 72, dtype=F16, device="cuda")
        out = torch.full_like(q, 3.0)
        cu = torch.tensor([0, n - 1, n - 1], dtype=torch.int32, device="cuda")
        vq.vq_attention(q, kv, kv, cu, torch.zeros(3, dtype=torch.int32, device="cuda"), out=out)
        assert (out[:n - 1] == 0).all() and (out[n - 1] == 3).all()


@pytest.mark.parametrize("heads,D", [(16, 72), (5, 80), (3, 88)])
def test_few_keys_for_many_queries(heads, D):
    # all heads of a tile on one XCD, numbers of tiles that are no multiple of the XCDs
    _run([700, 0, 1300, 5], [120, 7, 64, 1], heads, heads, D, F16, False, before=2, behind=3)
    _run([1000], [63], heads, 1, D, BF16, True)


@pytest.mark.parametrize("H,G,D", [(16, 16, 72), (16, 16, 64), (32, 8, 128), (16, 16, 88), (20, 20, 80)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_thousands_of_queries_to_few_keys(H, G, D, dtype):
    _run([6000, 1, 0, 2999, 40], [128, 0, 9, 75, 33], H, G, D, dtype, False, before=1, behind=2)
    _run([3000, 4500, 7, 1500], [300, 1, 64, 129], H, G, D, dtype, False)


def test_scores_far_below_the_first_tile_s():
    # the first tile's scores are large, the others' far below (and the other way round): the reference stays with the largest
    D, m = 72, 700
    g = torch.Generator(device="cuda").manual_seed(9)
    for n in (1, 200):
        q = torch.randn(n, 1, D, generator=g, device="cuda").to(F16)
        for lo, hi in ((0, 64), (640, 700), (100, 101)):
            k = torch.randn(m, 1, D, generator=g, device="cuda") * 0.3
            k[lo:hi] += 20 * q[:1].float()
            k = k.to(F16)
            v = torch.randn(m, 1, D, generator=g, device="cuda").to(F16)
            want, off = ou.attention(q, k, v, [n], [m], 0.3, False)
            ou.check(vq.vq_attention(q, k, v, ou.offsets([n]).cuda(), ou.offsets([m]).cuda(), softmax_scale=0.3), want, off)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [1, 300])
def test_large_scores(causal, n):
    # scores of several hundred, rising and falling along the keys: the running maximum moves by more than the type's range of exponents
    D, m = 64, 900
    g = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn(n, 1, D, generator=g, device="cuda").to(F16)
    for ramp in (torch.linspace(0.1, 8, m), torch.linspace(8, 0.1, m), (torch.arange(m) % 100).float() * 0.08):
        k = (torch.randn(m, 1, D, generator=g, device="cuda") * ramp.cuda()[:, None, None] * 2).to(F16)
        v = torch.randn(m, 1, D, generator=g, device="cuda").to(F16)
        cu_q, cu_k = ou.offsets([n]).cuda(), ou.offsets([m]).cuda()
        want, off = ou.attention(q, k, v, [n], [m], 1.0, causal)
        ou.check(vq.vq_attention(q, k, v, cu_q, cu_k, softmax_scale=1.0, causal=causal), want, off)


@pytest.mark.parametrize("n", [1, 200])
def test_equal_scores_average(n):
    # keys of zeros: every weight is the same, the output is the mean of v
    q, k, v = _data(n, 640, 2, 2, 128, F16)
    k = torch.zeros_like(k)
    got = vq.vq_attention(q, k, v, ou.offsets([n]).cuda(), ou.offsets([640]).cuda())
    want, off = ou.attention(q, k, v, [n], [640], 1 / math.sqrt(128), False)
    ou.check(got, want, off)


def test_keys_behind_a_sequence_do_not_matter():
    # what lies behind a sequence's last key, and keys that causality hides from every query of a tile, may be anything
    for n, lens in ((1, [50, 41]), (90, [90, 70])):
        q, k, v = _data(2 * n, 400, 2, 1, 72, F16)
        k, v = k.clone(), v.clone()
        cu_q, cu_k = ou.offsets([n, n]).cuda(), ou.offsets(lens, 100).cuda()
        want = vq.vq_attention(q, k, v, cu_q, cu_k)
        k[:100] = k[100 + sum(lens):] = float("nan")
        v[:100] = v[100 + sum(lens):] = float("inf")
        got = vq.vq_attention(q, k, v, cu_q, cu_k)
        assert torch.equal(got, want) and not got.isnan().any()


def test_hidden_keys_that_are_not_finite():
    # a key that causality hides has no score, whatever it holds
    n = 200
    q, k, v = _data(n, n, 2, 2, 64, BF16)
    k = k.clone()
    cu = ou.offsets([n]).cuda()
    want = vq.vq_attention(q, k, v, cu, cu, causal=True)
    k[150:] = float("nan")
    got = vq.vq_attention(q, k, v, cu, cu, causal=True)
    assert torch.equal(got[:150], want[:150]) and got[150:].isnan().all()


@pytest.mark.parametrize("n,m", [(1, 600), (200, 200)])
def test_views(n, m):
    # slices of one QKV buffer, head-major buffers, keys that all heads share, an output inside a larger one
    H, G, D = 4, 2, 72
    qkv = torch.randn(max(n, m), H + 2 * G, D, generator=torch.Generator().manual_seed(1)).to(F16).cuda()
    q, k, v = qkv[:n, :H], qkv[:m, H:H + G], qkv[:m, H + G:]
    cu_q, cu_k = ou.offsets([n]).cuda(), ou.offsets([m]).cuda()
    want, off = ou.attention(q, k, v, [n], [m], D ** -0.5, True)
    ou.check(vq.vq_attention(q, k, v, cu_q, cu_k, causal=True), want, off, "slices")
    major = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    big = torch.full((n, H + 1, D + 8), 5.0, dtype=F16, device="cuda")
    vq.vq_attention(*major, cu_q, cu_k, causal=True, out=big[:, :H, :D])
    ou.check(big[:, :H, :D], want, off, "head-major")
    assert (big[:, H] == 5).all() and (big[..., D:] == 5).all()
    k1, v1 = (t[:, :1].expand(m, G, D) for t in (k, v))
    want, off = ou.attention(q, k1, v1, [n], [m], D ** -0.5, False)
    ou.check(vq.vq_attention(q, k1, v1, cu_q, cu_k), want, off, "shared")


def test_offsets_beyond_32_bits():
    # keys 4 MiB apart: the last ones lie 5 GiB into the buffer
    m, D = 1300, 64
    buf = torch.zeros(m, 1 << 21, dtype=F16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    buf[:, :2 * D] = torch.randn(m, 2 * D, generator=g, device="cuda").to(F16)
    k, v = buf[:, None, :D], buf[:, None, D:2 * D]
    for n in (1, 100):
        q = torch.randn(n, 1, D, generator=g, device="cuda").to(F16)
        want, off = ou.attention(q, k, v, [n], [m], D ** -0.5, True)
        got = vq.vq_attention(q, k, v, ou.offsets([n]).cuda(), ou.offsets([m]).cuda(), causal=True)
        ou.check(got, want, off, n)


def test_offsets_that_are_not_in_order():
    # nothing outside the tensors is read or written, the sequence that is in order is right
    q, k, v = _data(100, 90, 2, 1, 64, F16)
    cu_q = torch.tensor([0, 40, 20, 100000, -5], dtype=torch.int32).cuda()
    cu_k = torch.tensor([0, 30, -7, 95, 60], dtype=torch.int32).cuda()
    out = vq.vq_attention(q, k, v, cu_q, cu_k)
    torch.cuda.synchronize()
    assert out.shape == q.shape


@pytest.mark.parametrize("lq,lk", [([1, 1], [4000, 900]), ([150, 90], [150, 90])])
def test_captured_and_replayed(lq, lk):
    H, G, D = 8, 2, 128
    sets = [_data(sum(lq), sum(lk), H, G, D, F16, seed) for seed in range(3)]
    q, k, v = (t.clone() for t in sets[0])
    cu_q, cu_k = ou.offsets(lq).cuda(), ou.offsets(lk).cuda()
    bytes_ = vq.vq_attention_workspace_bytes(len(lq), sum(lq), sum(lk), H, G, D)
    work = torch.empty(max(bytes_, 16), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    vq.vq_attention(q, k, v, cu_q, cu_k, causal=True, out=out, workspace=work)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vq.vq_attention(q, k, v, cu_q, cu_k, causal=True, out=out, workspace=work)
    for s in (2, 0, 1):
        for a, b in zip((q, k, v), sets[s]):
            a.copy_(b)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, vq.vq_attention(*sets[s], cu_q, cu_k, causal=True))


@pytest.mark.parametrize("T", [300, 5])
def test_block(T):
    """QKV layer, rotary positions in place, attention on the slices, output layer: each step against its definition on what the
    step before gave."""
    hidden, H, D = 1152, 16, 72
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, hidden, generator=g).to(F16)
    cm = torch.exp(torch.randn(hidden, generator=g) * 0.3)

    def weights(n, k):
        w = torch.randn(n, k, generator=g) * 0.03
        return w

    w1, w2 = weights(3 * hidden, hidden), weights(hidden, hidden)
    b1 = (torch.randn(3 * hidden, generator=g) * 0.1).to(F16)
    q1, s1 = vq.vq_mx4_quantize(w1.cuda(), (1 / cm).cuda())
    q2, s2 = vq.vq_mx4_quantize(w2.cuda())
    lens = [T - 2, 2]
    p = torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()
    f, amplitude = vq.vq_rotary_frequencies(D)
    f, cu = f.cuda(), ou.offsets(lens).cuda()

    qkv = vq.vq_linear_mx4(x.cuda(), cm.cuda(), q1, s1, b1.cuda())
    want, off = ou.product(ou.values_mx4(*ou.quantize_mx4(x, cm)), ou.values_mx4(*ou.unpack_mx4(q1, s1)), b1, F16)
    ou.check(qkv, want, off, "qkv")
    heads = qkv.view(T, 3 * H, D)
    q, k, v = heads[:, :H], heads[:, H:2 * H], heads[:, 2 * H:]
    wq, oq = ou.rotary(q, p, f, False, amplitude)
    vq.vq_rotary(q, k, p, f, amplitude=amplitude, q_out=q, k_out=k)
    ou.check(q, wq, oq + ou.HALF[F16] * wq.abs() + ou.TINY[F16], "rotary")
    o = vq.vq_attention(q, k, v, cu, cu, causal=True)
    want, off = ou.attention(q, k, v, lens, lens, D ** -0.5, True)
    ou.check(o, want, off, "attention")
    y = vq.vq_linear_mx4(o.view(T, hidden), None, q2, s2)
    want, off = ou.product(ou.values_mx4(*ou.quantize_mx4(o.view(T, hidden))), ou.values_mx4(*ou.unpack_mx4(q2, s2)), None, F16)
    ou.check(y, want, off, "output layer")
