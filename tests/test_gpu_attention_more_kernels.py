"""Attention in a window and behind a prefix: every kernel, head size and type at the lengths where its loops turn more than once."""
import pytest

import operator_util as ou
import test_gpu_attention_prefix as prefix
import test_gpu_attention_window as window
from test_gpu_attention_kernels import _lengths, _pairs

TILES, ROWS, ALONE = 0, 1, 2          # the kernels, as the library's choices number them
DIMS = [64, 72, 80, 96, 128]

# name: (kernel, whether the keys are divided, queries, keys, heads, heads of k and v, left, right, sinks, causal)
WINDOW = {
    "frames": (ALONE, False, [16] * 1030, [16] * 1030, 2, 2, 5, 3, 2, False),
    "ragged": (ALONE, False, _lengths(1, 1400, 0, 34, (70, 33, 0)), _lengths(2, 1400, 0, 90, (200, 65, 0)), 3, 3, 30, 10, 9, False),
    "short windows of long sequences": (ALONE, False, [1] * 1101, _lengths(3, 1100, 20, 300, (900,)), 6, 2, 20, 0, 4, True),
    "prompt among tokens": (ROWS, False, *_pairs([900] + [1] * 100, [900] + _lengths(5, 100, 1, 400)), 2, 2, 150, 0, 4, True),
    "tokens, grouped": (ROWS, False, [1] * 70 + [5], _lengths(6, 71, 0, 400), 8, 2, 200, 50, 70, False),
    "tokens, divided": (ROWS, True, [1] * 30 + [3], _lengths(7, 31, 1700, 2500), 4, 2, 1500, 0, 40, True),
    "prompts and tokens": (TILES, False, *_pairs([700, 333, 1, 1, 1], [700, 1000, 700, 1, 90]), 4, 2, 130, 0, 70, True),
    "both sides": (TILES, False, [900, 260, 0, 77], [900, 260, 30, 500], 3, 3, 200, 100, 0, False),
    "prompts, divided": (TILES, True, *_pairs([260, 1, 130], [3000, 2500, 1111]), 2, 1, 1200, 64, 200, False),
}
# name: (in parts, the kernel, whether the (own) keys are divided, whether the shared ones are, queries, keys, prefix, heads, heads of k and v)
PREFIX = {
    "tiles": (False, TILES, False, False, [500, 0, 130, 1], [300, 70, 30, 150], 130, 4, 2),
    "tiles, divided": (False, TILES, True, False, [260, 40], [70, 1000], 2000, 2, 1),
    "rows": (False, ROWS, False, False, [1] * 50 + [9, 0], _lengths(1, 51, 0, 90, (300,)), 130, 4, 2),
    "rows, divided": (False, ROWS, True, False, [1, 3, 2], [50, 0, 700], 3000, 4, 2),
    "parts by rows": (True, ROWS, False, True, [1] * 10, _lengths(2, 10, 0, 300), 9000, 3, 3),
    "parts by rows, divided": (True, ROWS, True, True, [1] * 8, _lengths(3, 8, 800, 1500), 11000, 4, 4),
    "parts by tiles": (True, TILES, False, True, [1] * 60 + [3, 0], _lengths(4, 61, 0, 200, (700,)), 5000, 8, 2),
    "parts by tiles, many sequences": (True, TILES, False, True, [1] * 129 + [40], _lengths(8, 130, 0, 60), 5001, 8, 2),
    "parts by tiles, whole": (True, TILES, False, False, _lengths(5, 700, 0, 3, (40,)), _lengths(6, 700, 0, 40, (100,)), 130, 8, 2),
    "parts by tiles, divided": (True, TILES, True, True, [7] * 12, _lengths(7, 12, 600, 900), 4001, 12, 2),
}


@pytest.mark.gpu
@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("name", WINDOW)
def test_window(name, D):
    _, _, lq, lk, H, G, left, right, sinks, causal = WINDOW[name]
    window._run(lq, lk, H, G, D, ou.F16, left, right, sinks, causal, before=2, behind=3)
    window._run(lq, lk, H, G, D, ou.BF16, left, right, sinks, causal)


@pytest.mark.gpu
@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("name", PREFIX)
def test_prefix(name, D):
    *_, lq, lk, P, H, G = PREFIX[name]
    prefix._run(lq, lk, P, H, G, D, ou.F16, D % 3 == 0, before=2, behind=3)
    prefix._run(lq, lk, P, H, G, D, ou.BF16, D % 3 != 0)
