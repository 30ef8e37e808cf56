"""Rotary positions of several axes and norms: every kernel, several tokens a workgroup at head counts that are no powers of two, and rows far apart,
against the formulas in 64 bits."""
import pytest
import torch

import paper_2406_02540_amd as vq
import more_operator_util as mu
import operator_util as ou
from test_gpu_rotary_axes import PAIRINGS, _angles, _views

F16, BF16 = ou.F16, ou.BF16

# tokens, heads, heads of k, head_dim, pairs of every axis: (channels that keep together on their way to their partners with halves and with each axis' own
# halves, tokens of a workgroup)
SEVERAL = {(7257, 5, 1, 96, (4, 10, 10)): (8, 2, 5), (2501, 12, 3, 64, (31,)): (1, 1, 2), (2501, 5, 2, 128, (16, 24, 24)): (8, 8, 2),
           (9001, 3, 1, 64, (8, 24)): (8, 8, 6), (6000, 1, 1, 8, (1, 2)): (1, 1, 4), (5003, 2, 1, 40, (4, 8)): (4, 4, 4),
           (3001, 11, 0, 24, (6,)): (2, 2, 2), (1700, 9, 5, 56, (20, 4)): (8, 4, 2), (16001, 3, 3, 16, (4, 4)): (8, 4, 8)}
# pairs of every axis and how they lie, for heads of 64: the channels that keep together
FAR = {((8, 24), "halves"): 8, ((4, 8), "axis_halves"): 4, ((2, 20), "axis_halves"): 2, ((31,), "halves"): 1, ((8, 3, 4), "neighbours"): 0}
APART = 2**29 + 8        # values from head to head: three heads span more than 2^31 bytes


def _check(got, x, w, b, kind, p, f, sections, pairing, what):
    x = x.double().cpu()
    want, off = (x, torch.zeros_like(x)) if kind is None else mu.norm(x, w, b, kind, 1e-6)
    want, off = mu.turn(want, off, p, f, sections, pairing, 1.5)
    ou.check(got, want, mu.rounded(want, off, got.dtype), what)


def _call(kind, q, k, vectors, p, f, sections, pairing, **out):
    if kind is None:
        return vq.vq_rotary_axes(q, k, p, f, sections, pairing=pairing, amplitude=1.5, **out)
    qw, kw, qb, kb = vectors
    return vq.vq_norm_rotary(q, k, qw, kw if k is not None else None, qb, kb if k is not None else None, norm=kind, eps=1e-6, positions=p, inv_freq=f,
                             sections=sections, pairing=pairing, amplitude=1.5, **out)


def _vectors(D):
    g = torch.Generator().manual_seed(D)
    return [(1 + 0.3 * torch.randn(D, generator=g)).cuda() for _ in range(2)] + [0.2 * torch.randn(D, generator=g).cuda() for _ in range(2)]


@pytest.mark.gpu
@pytest.mark.parametrize("pairing", PAIRINGS)
@pytest.mark.parametrize("T,H,G,D,sections", SEVERAL)
def test_several_tokens_a_workgroup(T, H, G, D, sections, pairing):
    p, f = _angles(T, sections)
    for n, kind in enumerate((None, "rms", "layer")):
        dtype = (F16, BF16)[(n + PAIRINGS.index(pairing)) % 2]
        _, q, k = _views(T, H, G, D, dtype, spread=kind is not None)
        k = k if G else None
        vectors = _vectors(D)
        if kind == "rms":
            vectors[2:] = None, None
        qo, ko = _call(kind, q, k, vectors, p, f, sections, pairing)
        _check(qo, q, vectors[0], vectors[2], kind, p, f, sections, pairing, (kind, "q"))
        if G:
            _check(ko, k, vectors[1], vectors[3], kind, p, f, sections, pairing, (kind, "k"))


@pytest.mark.gpu
def test_ragged_tokens_of_wide_heads():
    T, H, G, D, sections = 7257, 20, 4, 96, (4, 10, 10)
    _, q, k = _views(T, H, G, D, BF16, spread=True)
    p, f = _angles(T, sections)
    vectors = _vectors(D)
    qo, ko = _call("layer", q, k, vectors, p, f, sections, "axis_halves")
    _check(qo, q, vectors[0], vectors[2], "layer", p, f, sections, "axis_halves", "q")
    _check(ko, k, vectors[1], vectors[3], "layer", p, f, sections, "axis_halves", "k")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_heads_more_than_32_bits_apart(dtype):
    T, H, D = 3, 3, 64
    room = torch.empty((H - 1) * APART + 8 * T * D, dtype=dtype, device="cuda")
    at = [n * APART for n in range(H)]
    for n in at:
        room[n:n + 8 * T * D] = 7
    far = room.as_strided((T, H, D), (2 * D, APART, 1))                  # every other row is another's
    _, q, k = _views(T, H, 1, D, dtype, spread=True)
    vectors = _vectors(D)
    for (sections, pairing) in FAR:
        p, f = _angles(T, sections)
        for kind in (None, "rms", "layer"):
            what = (sections, pairing, kind)
            want, want_k = _call(kind, q, k, vectors, p, f, sections, pairing)
            _check(want, q, vectors[0], vectors[2], kind, p, f, sections, pairing, what)
            far.fill_(5)
            got, got_k = _call(kind, q, k, vectors, p, f, sections, pairing, q_out=far)
            assert got is far and torch.equal(far, want) and torch.equal(got_k, want_k), what
            far.copy_(q)
            got, got_k = _call(kind, far, k, vectors, p, f, sections, pairing)
            assert torch.equal(got, want) and torch.equal(got_k, want_k), what
            _call(kind, far, k, vectors, p, f, sections, pairing, q_out=far)
            assert torch.equal(far, want), what
            # and as k
            far.copy_(q)
            same = [vectors[1], vectors[0], vectors[3], vectors[2]]
            got_k, got = _call(kind, k, far, same, p, f, sections, pairing)
            assert torch.equal(got, want) and torch.equal(got_k, want_k), what
    for n in at:
        rows = room[n:n + 8 * T * D].view(-1, D)
        assert (rows[1:2 * T:2] == 7).all() and (rows[2 * T:] == 7).all()


@pytest.mark.gpu
def test_heads_just_within_32_bits():
    # the last channel of the last head ends below 2^31 bytes: the kernels with 32-bit offsets
    T, H, D, sections = 2, 2, 64, (8, 24)
    room = torch.empty(2**30, dtype=F16, device="cuda")
    far = room.as_strided((T, H, D), (D, 2**30 - 2 * D, 1))
    _, q, k = _views(T, H, 1, D, F16)
    p, f = _angles(T, sections)
    for pairing in PAIRINGS:
        want = vq.vq_rotary_axes(q, None, p, f, sections, pairing=pairing)[0]
        far.copy_(q)
        vq.vq_rotary_axes(far, None, p, f, sections, pairing=pairing, q_out=far)
        assert torch.equal(far, want)
