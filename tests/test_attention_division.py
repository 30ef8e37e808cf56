"""How keys are divided among workgroups where the sequences' own lengths decide: windows that do not shorten them and short prefixes as vq_attention does."""
import ctypes
import os

import pytest

from paper_2406_02540_amd import binding, build

# sequences, queries, keys, heads, heads of k and v
BATCHES = [(16, 16, 16 * 12000, 32, 8), (48, 48, 48 * 12362, 32, 8), (64, 64, 64 * 4096, 32, 8), (32, 32, 32 * 2870, 32, 8), (4, 9, 4 * 17651, 32, 8),
           (16, 16, 16 * 11000, 16, 16), (2, 700, 2 * 9000, 8, 2), (100, 100, 100 * 400, 8, 8)]


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)


def _attention(*sizes):
    out = (ctypes.c_int * 2)()
    binding.lib().vq_internal_attention_choice(*sizes, out)
    return tuple(out)


def _window(sizes, causal, left, right, sinks):
    out = (ctypes.c_int * 2)()
    binding.lib().vq_internal_attention_window_choice(*sizes, causal, left, right, sinks, out)
    return tuple(out)


@pytest.mark.parametrize("sizes", BATCHES)
def test_windows_that_leave_the_sequences_as_they_are(sizes):
    average = sizes[2] // sizes[0]
    for causal, left, right, sinks in ((1, -1, 0, 0), (0, -1, -1, 0), (0, -1, 5, 4), (0, 5, -1, 0), (1, 2 * average, 0, 0), (1, 2**31 - 1, 2**31 - 1, 7),
                                       (0, average, average, 0)):
        assert _window(sizes, causal, left, right, sinks) == _attention(*sizes), (causal, left, right, sinks)


def test_windows_that_make_them_equal():
    # a workgroup a CU for the keys of a window, in 2 parts or 8 or one
    assert _window((48, 48, 48 * 12362, 32, 8), 1, 4095, 0, 4) == (1, 1)
    assert _window((4, 4, 4 * 17651, 32, 8), 1, 4095, 0, 4) == (1, 3)
    assert _window((64, 64, 64 * 8192, 32, 8), 1, 4095, 0, 4) == (1, 0)
    assert _window((32, 32, 32 * 2870, 32, 8), 1, 2870, 0, 4) == (1, 0)


def test_a_division_pays_for_its_join():
    # 512 keys in two parts take longer than undivided, 1000 do not
    assert _window((16, 16, 16 * 8192, 32, 8), 1, 511, 0, 0) == (1, 0)
    assert _window((48, 48, 48 * 8192, 32, 8), 1, 599, 0, 0) == (1, 0)
    assert _window((16, 16, 16 * 8192, 32, 8), 1, 999, 0, 0) == (1, 1)


def _prefix(sequences, Tq, P, Tk, H, G, D):
    out = (ctypes.c_int * 4)()
    binding.lib().vq_internal_attention_prefix_choice(sequences, Tq, P, Tk, H, G, D, out)
    return tuple(out)


@pytest.mark.parametrize("sizes", BATCHES)
def test_prefixes_that_leave_the_sequences_as_they_are(sizes):
    sequences, Tq, Tk, H, G = sizes
    assert _prefix(sequences, Tq, 0, Tk, H, G, 128) == (0, *_attention(*sizes), 0)
    P = 16 if sequences < 100 else 4
    assert _prefix(sequences, Tq, P, Tk, H, G, 128) == (0, *_attention(sequences, Tq, Tk + P * sequences, H, G), 0)


def test_prefixes_that_are_most_of_the_keys():
    assert _prefix(2, 2, 3000, 400, 8, 2, 64) == (0, 1, 3, 0)
    assert _prefix(3, 6, 2000, 900, 32, 8, 64) == (0, 1, 3, 0)


@pytest.mark.parametrize("sizes", BATCHES[:4] + [(32, 32, 32 * 2000, 32, 8), (24, 48, 24 * 5000, 16, 8)])
def test_own_keys_behind_many_shared_ones(sizes):
    sequences, Tq, Tk, H, G = sizes
    in_parts, _, own, _ = _prefix(sequences, Tq, 4096, Tk, H, G, 128)
    assert in_parts and own == min(_attention(*sizes)[1], 5)


def test_parts_of_many_rows_are_few():
    assert _prefix(64, 6400, 9000, 64 * 2000, 8, 8, 128)[::2] == (1, 0)


def _own_items(sequences, Tq, P, Tk, H, G, D):
    return binding.lib().vq_internal_attention_prefix_own_items(sequences, Tq, P, Tk, H, G, D)


def test_rows_with_their_own_keys_are_no_chain():
    # sequences of more than a token: a workgroup a head for every block of 64 rows, whatever sequence it is of
    for sequences, tokens, H, G, D in ((64, 1963, 32, 8, 128), (16, 812, 16, 8, 64), (61, 460, 8, 2, 64), (200, 3200, 16, 8, 128)):
        sizes = sequences, tokens, 8192, 100 * sequences, H, G, D
        assert _prefix(*sizes)[0] == 1
        assert _own_items(*sizes) == tokens * (H // G) // 64 + sequences
    # single tokens: one for every sequence
    assert _prefix(64, 64, 8192, 6400, 32, 8, 128)[0] == 1 and _own_items(64, 64, 8192, 6400, 32, 8, 128) == 64


def test_the_largest_sizes():
    # (their products with the bytes of a key pass 63 bits; views may repeat one key)
    most = 2**31 - 768
    for sequences in (1 << 22, 1 << 23, (1 << 23) + 999):
        for tokens in (sequences, 2 * sequences):
            assert _prefix(sequences, tokens, most, 0, 1, 1, 128)[0] == 1, sequences
    bytes_of = binding.lib().vq_attention_prefix_workspace_bytes
    assert [bytes_of(2**31 - 1, tokens, most, 0, G, G, 128) for G in (1, 8, 1 << 16) for tokens in (1, 2**31 // G - 256)] == [0] * 6
