"""The sizes that include/vq.h allows for attention, in a window and behind a prefix: the refusals of larger launches begin beyond them.  CPU only: a call that
gets as far as the device's check was accepted."""
import ctypes
import os
import random

import pytest

from paper_2406_02540_amd import binding, build

A = 0x10000
P, F = ctypes.c_void_p, ctypes.c_float
ARCH = 6
MOST = 2**31 - 256


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    return binding.lib()


def _calls(lib, B, Tq, P_, Tk, H, G, D):
    q, k = (H * D, D), (G * D, D)
    eight, twelve = (ctypes.c_int64 * 8)(*q, *k, *k, *q), (ctypes.c_int64 * 12)(*q, *k, *k, *k, *k, *q)
    end = (P(A), 1 << 62, None)
    p = P(A)
    yield "attention", 8, lambda: lib.vq_attention(p, p, p, P(1 << 50), 0, p, p, B, Tq, Tk, H, G, D, eight, F(0.1), 1, *end)
    yield "window", 64, lambda: lib.vq_attention_window(p, p, p, P(1 << 50), 0, p, p, B, Tq, Tk, H, G, D, eight, F(0.1), 1, 100, 0, 4, *end)
    yield "prefix", 8, lambda: lib.vq_attention_prefix(p, p, p, p, p, P(1 << 50), 0, p, p, B, Tq, P_, Tk, H, G, D, twelve, F(0.1), 1, *end)


def _check(lib, B, Tq, P_, Tk, H, G, D):
    for name, rounded, call in _calls(lib, B, Tq, P_, Tk, H, G, D):
        if Tq * H / 128 + (B + rounded) * G < 2**24:
            assert call() == ARCH, (name, B, Tq, P_, Tk, H, G, D)


def test_random_sizes(lib):
    r = random.Random(7)
    for _ in range(20000):
        G = r.choice((1, 1, 2, 3, 7, 8, 64))
        H = G * r.choice((1, 2, 4, 7, 48))
        Tq = int(2 ** r.uniform(0, 31)) % (MOST // H) + 1
        B = int(2 ** r.uniform(0, 24)) // G + 1
        if r.random() < 0.5:                      # from single tokens to 200 rows a sequence
            B = max(1, int(Tq / (2 ** r.uniform(0, 7.6) * G / H + 1)))
        prefix = int(2 ** r.uniform(0, 30))
        Tk = min(int(2 ** r.uniform(0, 31)), MOST - prefix)
        _check(lib, B, Tq, prefix, Tk, H, G, r.choice((8, 64, 72, 128)))


def test_many_rows_in_parts(lib):
    # 128 rows a sequence behind many shared keys, one head of k and eight
    for H, G in ((1, 1), (8, 8), (8, 1), (2, 2)):
        for rows in (2**27, 2**28, 2**29, 2**30, MOST):
            Tq = rows // H
            for a_sequence in (1, 32, 33, 100, 128):
                _check(lib, max(1, Tq * (H // G) // a_sequence), Tq, 8192, 0, H, G, 8)
