"""Rotary positions of several axes, and norms of heads with them, against the formulas in 64 bits."""
import ctypes

import pytest
import torch

import paper_2406_02540_amd as vq
from paper_2406_02540_amd.binding import lib
import more_operator_util as mu
import operator_util as ou

pytestmark = pytest.mark.gpu
F16, BF16 = ou.F16, ou.BF16

# tokens, heads, heads of k, head_dim, pairs of every axis
SHAPES = [(1, 1, 1, 8, (1,)), (1, 32, 8, 128, (16, 24, 24)), (7, 3, 1, 64, (10, 22)), (100, 16, 16, 72, (8, 14, 14)), (33, 5, 5, 80, (1, 2, 3, 4)),
          (513, 4, 2, 96, (48,)), (3001, 16, 16, 72, (18, 18)), (5, 2, 1, 72, (3, 6)), (1100, 32, 8, 128, (62,)), (9, 3, 3, 8, (1, 1, 1, 1)),
          (65, 4, 1, 64, (31,)), (257, 1, 1, 120, (17, 20, 23)), (40, 70, 3, 24, (4, 4))]
PAIRINGS = ["halves", "neighbours", "axis_halves"]


def _views(T, H, G, D, dtype, seed=0, spread=False):
    g = torch.Generator().manual_seed(seed + 7 * T + D)
    x = torch.randn(T, H + 2 * G, D, generator=g)
    if spread:
        x = x * torch.exp(2 * torch.randn(T, H + 2 * G, 1, generator=g)) + 0.5 * torch.randn(1, 1, D, generator=g)
    buf = x.to(dtype).cuda()
    return buf, buf[:, :H], buf[:, H:H + G]


def _angles(T, sections, seed=0, far=True):
    g = torch.Generator().manual_seed(T + seed)
    top = 1 << 20 if far else 300
    p = torch.randint(-top, top, (len(sections), T), generator=g, dtype=torch.int32).cuda()
    f = torch.cat([vq.vq_rotary_frequencies(2 * n)[0] for n in sections]).cuda()
    return p, f


def _check_turned(got, x, p, f, sections, pairing, amplitude, what):
    x = x.double().cpu()
    want, off = mu.turn(x, torch.zeros_like(x), p, f, sections, pairing, amplitude)
    ou.check(got, want, mu.rounded(want, off, got.dtype), what)
    R = 2 * sum(sections)
    assert torch.equal(got.cpu().double()[..., R:], x[..., R:])


@pytest.mark.parametrize("T,H,G,D,sections", SHAPES)
@pytest.mark.parametrize("pairing", PAIRINGS)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_axes(T, H, G, D, sections, pairing, dtype):
    buf, q, k = _views(T, H, G, D, dtype)
    kept = buf.clone()
    p, f = _angles(T, sections)
    qo, ko = vq.vq_rotary_axes(q, k, p, f, sections, pairing=pairing, amplitude=1.25)
    assert torch.equal(buf, kept) and qo.is_contiguous() and ko.is_contiguous()
    _check_turned(qo, q, p, f, sections, pairing, 1.25, "q")
    _check_turned(ko, k, p, f, sections, pairing, 1.25, "k")
    # in place: the same numbers, the rest of the buffer as it was
    vq.vq_rotary_axes(q, k, p, f, list(sections), pairing=pairing, amplitude=1.25, q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(buf[:, H + G:], kept[:, H + G:])
    alone, none = vq.vq_rotary_axes(kept[:, :H], None, p, f, sections, pairing=pairing, amplitude=1.25)
    assert none is None and torch.equal(alone, qo)


@pytest.mark.parametrize("pairing,interleaved", [("halves", False), ("neighbours", True), ("axis_halves", False)])
def test_one_axis_is_vq_rotary(pairing, interleaved):
    _, q, k = _views(50, 4, 2, 64, F16)
    p, f = _angles(50, (24,))
    # (each within the same distance of the formula: products and sum round once here and three times there)
    for x, a, b in zip((q, k), vq.vq_rotary_axes(q, k, p, f, (24,), pairing=pairing), vq.vq_rotary(q, k, p[0], f, interleaved=interleaved)):
        x = x.double().cpu()
        want, off = mu.turn(x, torch.zeros_like(x), p, f, (24,), pairing, 1.0)
        assert ((a.double() - b.double()).abs().cpu() <= 2 * mu.rounded(want, off, F16)).all()


@pytest.mark.parametrize("T,H,G,D,sections", SHAPES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_norm(T, H, G, D, sections, kind, dtype):
    buf, q, k = _views(T, H, G, D, dtype, spread=True)
    kept = buf.clone()
    g = torch.Generator().manual_seed(D)
    vectors = [(1 + 0.3 * torch.randn(D, generator=g)).cuda(), (1 + 0.3 * torch.randn(D, generator=g)).cuda(),
               0.2 * torch.randn(D, generator=g).cuda(), 0.2 * torch.randn(D, generator=g).cuda()]
    p, f = _angles(T, sections)
    for pairing, use in zip(PAIRINGS + [None], ((1, 1, 1, 1), (1, 1, 0, 0), (0, 0, 0, 0), (1, 0, 0, 1))):
        qw, kw, qb, kb = (v if u else None for v, u in zip(vectors, use))
        turn = {} if pairing is None else {"positions": p, "inv_freq": f, "sections": sections, "pairing": pairing, "amplitude": 0.75}
        got = vq.vq_norm_rotary(q, k, qw, kw, qb, kb, norm=kind, eps=1e-5, **turn)
        assert torch.equal(buf, kept)
        for name, x, y, w, b in (("q", q, got[0], qw, qb), ("k", k, got[1], kw, kb)):
            want, off = mu.norm(x, w, b, kind, 1e-5)
            if pairing is not None:
                want, off = mu.turn(want, off, p, f, sections, pairing, 0.75)
            ou.check(y, want, mu.rounded(want, off, dtype), (name, pairing, use))
        alone, none = vq.vq_norm_rotary(q, None, qw, None, qb, norm=kind, eps=1e-5, **turn)
        assert none is None and torch.equal(alone, got[0])
        work = buf.clone()
        vq.vq_norm_rotary(work[:, :H], work[:, H:H + G], qw, kw, qb, kb, norm=kind, eps=1e-5, q_out=work[:, :H], k_out=work[:, H:H + G], **turn)
        assert torch.equal(work[:, :H], got[0]) and torch.equal(work[:, H:H + G], got[1]) and torch.equal(work[:, H + G:], buf[:, H + G:])


def test_positions_at_the_ends_of_their_range():
    ends = [0, 1, -1, 2**31 - 1, -2**31, 2**30 + 1]
    p = torch.tensor([ends, ends[::-1], [5] * 6], dtype=torch.int32).cuda()
    _, q, k = _views(6, 2, 1, 64, F16)
    sections = (12, 12, 8)
    _, f = _angles(6, sections)
    for pairing in PAIRINGS:
        qo, ko = vq.vq_rotary_axes(q, k, p, f, sections, pairing=pairing)
        _check_turned(qo, q, p, f, sections, pairing, 1.0, "far")
        _check_turned(ko, k, p, f, sections, pairing, 1.0, "far")


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_heads_of_zeros_of_equal_values_and_that_are_not_finite(kind):
    T, H, D = 20, 6, 72
    _, q, _ = _views(T, H, 1, D, F16)
    q = q.clone()
    q[3, 2] = 0
    q[4, 1] = 2.5
    q[5, 0] = 6e4
    q[6, 3] = 2.0 ** -24
    want = vq.vq_norm_rotary(q, None, norm=kind, eps=1e-6)[0]
    w, off = mu.norm(q, None, None, kind, 1e-6)
    ou.check(want, w, mu.rounded(w, off, F16))
    assert (want[3, 2] == 0).all() and (kind == "rms" or (want[4, 1] == 0).all())
    bad = q.clone()
    bad[7, 4, 3], bad[8, 5, 71], bad[0, 0, 0] = float("nan"), float("inf"), float("-inf")
    got = vq.vq_norm_rotary(bad, None, norm=kind, eps=1e-6)[0]
    hit = torch.zeros(T, H, dtype=torch.bool, device="cuda")
    hit[7, 4] = hit[8, 5] = hit[0, 0] = True
    assert torch.equal(got[~hit], want[~hit])


def test_views_of_other_orders():
    T, H, D, sections = 50, 4, 64, (8, 12, 12)
    base = torch.randn(H, T, D, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    q = base.transpose(0, 1)                                  # heads outermost in memory
    one = torch.randn(T, 1, D, generator=torch.Generator().manual_seed(2)).to(BF16).cuda().expand(T, 3, D)
    p, f = _angles(T, sections, far=False)
    wide = torch.full((T, H + 1, D + 16), 7.0, dtype=BF16, device="cuda")
    for pairing in PAIRINGS:
        out = torch.empty(H, T, D, dtype=BF16, device="cuda").transpose(0, 1)
        qo, ko = vq.vq_rotary_axes(q, one, p, f, sections, pairing=pairing, q_out=out)
        assert qo is out
        _check_turned(out, q, p, f, sections, pairing, 1.0, "head-major")
        _check_turned(ko, one, p, f, sections, pairing, 1.0, "shared")
        vq.vq_norm_rotary(q, None, positions=p, inv_freq=f, sections=sections, pairing=pairing, q_out=wide[:, :H, 8:8 + D])
        want, off = mu.turn(*mu.norm(q, None, None, "rms", 1e-6), p, f, sections, pairing, 1.0)
        ou.check(wide[:, :H, 8:8 + D], want, mu.rounded(want, off, BF16), "inside a larger one")
        assert (wide[:, H] == 7).all() and (wide[:, :, :8] == 7).all() and (wide[:, :, 8 + D:] == 7).all()


def test_no_tokens():
    q = torch.empty(0, 4, 64, dtype=F16, device="cuda")
    p, f = torch.empty(2, 0, dtype=torch.int32, device="cuda"), torch.ones(16, device="cuda")
    assert vq.vq_rotary_axes(q, q, p, f, (8, 8))[0].shape == (0, 4, 64)
    assert vq.vq_norm_rotary(q, None)[0].shape == (0, 4, 64)


def test_what_belongs_to_k_is_not_looked_at_without_it():
    T, H, D = 5, 4, 64
    buf, q, _ = _views(T, H, 1, D, F16)
    w = torch.rand(D + 4, device="cuda") + 0.5
    want = vq.vq_norm_rotary(q, None, w[:D])[0]
    got = torch.empty_like(want)
    other = ctypes.c_void_p(w.data_ptr() + 4)           # (with heads of k its weights and biases would be refused)
    strides = (ctypes.c_int64 * 8)(*q.stride()[:2], *got.stride()[:2], 0, 0, 0, 0)
    P, stream = ctypes.c_void_p, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert lib().vq_norm_rotary(P(q.data_ptr()), P(got.data_ptr()), None, None, 0, 0, ctypes.c_float(1e-6), P(w.data_ptr()), None, other, other, None,
                                None, ctypes.c_float(1), 0, 0, None, T, H, 0, D, strides, stream) == 0
    assert torch.equal(got, want)


@pytest.mark.parametrize("T", [1, 200, 4000])
def test_captured_and_replayed(T):
    buf, q, k = _views(T, 8, 2, 72, F16, spread=True)
    sections = (8, 14, 14)
    p, f = _angles(T, sections, far=False)
    w = torch.rand(72, device="cuda") + 0.5
    qo, ko = torch.empty(T, 8, 72, dtype=F16, device="cuda"), torch.empty(T, 2, 72, dtype=F16, device="cuda")

    def call(**out):
        return vq.vq_norm_rotary(q, k, w, w, positions=p, inv_freq=f, sections=sections, pairing="neighbours", **out)

    call(q_out=qo, k_out=ko)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(q_out=qo, k_out=ko)
    for shift in (1000, 0, 77):
        p.copy_(torch.randint(0, 500, p.shape, dtype=torch.int32) + shift)
        buf.mul_(0.9)
        qo.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = call()
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])


def test_on_another_stream():
    _, q, k = _views(3000, 16, 16, 72, F16)
    p, f = _angles(3000, (36,))
    want = vq.vq_rotary_axes(q, k, p, f, (36,))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        inner = vq.vq_rotary_axes(q, k, p, f, (36,))
    given = vq.vq_rotary_axes(q, k, p, f, (36,), stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b, c in zip(want, inner, given):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_more_values_than_32_bits_count():
    # 33.6 million tokens of 8 heads of 8 channels: 2^31 values, 2^30 pairs
    T, H, D = (1 << 25) + 3, 8, 8
    q = torch.zeros(T, H, D, dtype=F16, device="cuda")
    at = torch.tensor([0, 1, T // 2, (1 << 24) + 1, T - 2, T - 1], device="cuda")
    q[at] = torch.randn(6, H, D, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(F16)
    p = torch.arange(2 * T, dtype=torch.int32, device="cuda").view(2, T)
    f = torch.tensor([1.0, 0.1, 0.5, 0.02], device="cuda")
    vq.vq_norm_rotary(q[at].contiguous(), None)
    small = vq.vq_rotary_axes(q[at].contiguous(), None, p[:, at].contiguous(), f, (2, 2))[0]
    normed = vq.vq_norm_rotary(q[at].contiguous(), None, positions=p[:, at].contiguous(), inv_freq=f, sections=(2, 2))[0]
    out = torch.full_like(q, 3.0)
    vq.vq_rotary_axes(q, None, p, f, (2, 2), q_out=out)
    assert torch.equal(out[at], small) and int((out == 0).sum()) >= (T - 6) * H * D
    vq.vq_norm_rotary(q, None, positions=p, inv_freq=f, sections=(2, 2), q_out=out)
    assert torch.equal(out[at], normed) and int((out == 0).sum()) >= (T - 6) * H * D
