"""Attention: every kernel, head size and type at the lengths where its loops turn more than once, batches that mix a prompt with single
tokens, and offsets that are out of order or outside the tensors."""
import random

import pytest
import torch

import paper_2406_02540_amd as vq
import operator_util as ou
from test_gpu_attention import _data, _run

TILES, ROWS, ALONE = 0, 1, 2          # the kernels, as vq_internal_attention_choice() numbers them


def _lengths(seed, n, lo, hi, more=()):
    r = random.Random(seed)
    lens = [r.randint(lo, hi) for _ in range(n)] + list(more)
    r.shuffle(lens)
    return lens


def _pairs(queries, keys):
    """Queries and keys in one order."""
    both = list(zip(queries, keys))
    random.Random(len(both)).shuffle(both)
    return [list(x) for x in zip(*both)]


# name: (kernel, whether the keys are divided, queries, keys, heads, heads of k and v)
CASES = {
    # a wavefront a sequence: frames of a video, ragged ones with empty sequences, several blocks of rows and of keys, grouped heads
    "frames": (ALONE, False, [16] * 1030, [16] * 1030, 2, 2),
    "ragged": (ALONE, False, _lengths(1, 1400, 0, 34, (70, 33, 0)), _lengths(2, 1400, 0, 90, (200, 65, 0)), 3, 3),
    "grouped": (ALONE, False, _lengths(3, 1100, 0, 12, (90,)), _lengths(4, 1100, 0, 100, (3,)), 6, 2),
    "one long among short": (ALONE, False, *_pairs([300] + [3] * 1099, [500] + [5] * 1099), 2, 2),
    # four wavefronts a sequence: a prompt among single tokens, and with the keys divided
    "prompt among tokens": (ROWS, False, *_pairs([900] + [1] * 100, [900] + _lengths(5, 100, 1, 400)), 2, 2),
    "prompt among tokens, grouped": (ROWS, False, *_pairs([201] + [1] * 100, [333] + _lengths(6, 100, 0, 400)), 8, 2),
    "prompt among tokens, divided": (ROWS, True, *_pairs([600] + [1] * 40, [640] + _lengths(7, 40, 700, 2500)), 2, 2),
    # tiles: the same with shorter batches, and with the keys divided
    "prompts and tokens": (TILES, False, *_pairs([500, 333, 1, 1, 1], [500, 1000, 700, 1, 90]), 4, 2),
    "prompts and tokens, divided": (TILES, True, *_pairs([260, 1, 130], [3000, 2500, 1111]), 2, 1),
}
DIMS = [64, 72, 80, 96, 128]


@pytest.mark.gpu
@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("name", CASES)
def test_kernels(name, D):
    _, _, lq, lk, H, G = CASES[name]
    _run(lq, lk, H, G, D, ou.F16, D % 3 == 0, before=2, behind=3)
    _run(lq, lk, H, G, D, ou.BF16, D % 3 != 0)


# Offsets in front of the tensors, behind them and falling: a sequence is what lies within the tensors, falling offsets are no rows.
BAD = [([-20, 40, 100000, 300, 120], [-7, 30, 200000, 95, 1 << 30], (40, 60)), ([0, 40, 20, -5, -7], [0, 30, 10, -4, -9], (40, 0))]
# (heads, heads of k and v, keys, kernel, divided)
BAD_SHAPES = [(2, 1, 90, TILES, False), (1, 1, 90, ROWS, False), (1, 1, 4000, ROWS, True), (6, 2, 4000, TILES, True)]


@pytest.mark.gpu
@pytest.mark.parametrize("cu_q,cu_k,rows", BAD)
@pytest.mark.parametrize("H,G,Tk", [s[:3] for s in BAD_SHAPES])
def test_offsets_outside_the_tensors(cu_q, cu_k, rows, H, G, Tk):
    Tq, D, divided = 100, 64, Tk > 90
    room = torch.full((Tq + 64, H, D), 5.0, dtype=ou.F16, device="cuda")
    q, k, v = _data(Tq, Tk, H, G, D, ou.F16)
    cu = [torch.tensor(c, dtype=torch.int32).cuda() for c in (cu_q, cu_k)]
    vq.vq_attention(q, k, v, *cu, out=room[32:32 + Tq])
    assert (room[:32] == 5).all() and (room[32 + Tq:] == 5).all()
    if divided and cu_q[-1] < cu_q[0] + Tq:      # (the parts are joined for the rows from the first offset to the last)
        return
    clamped = [[min(max(c, 0), t) for c in cu] for cu, t in ((cu_q, Tq), (cu_k, Tk))]
    lk = [max(b - a, 0) for a, b in zip(clamped[1], clamped[1][1:])][:2]
    want, off = ou.attention(q, k, v, rows, lk, D ** -0.5, False)
    ou.check(room[32:32 + sum(rows)], want[:sum(rows)], off[:sum(rows)], (cu_q, cu_k))
