"""Which kernel rotary positions of several axes and norms reach, and what its workgroups take: the shapes of the GPU tests reach every one."""
import ctypes
import os

import pytest

from paper_2406_02540_amd import binding, build

pytest.importorskip("torch")

HALVES, NEIGHBOURS, AXIS_HALVES = 0, 1, 2


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)


def choice(norm, has_bias, pairing, T, H, G, D, sections, strides=None):
    """(channels that keep together, whether offsets are of 64 bits, tokens of a workgroup, heads of a workgroup)."""
    out = (ctypes.c_int * 4)()
    s = strides or ((H + 2 * G) * D, D, H * D, D, (H + 2 * G) * D, D, G * D, D)
    binding.lib().vq_internal_rotary_axes_choice(norm, has_bias, pairing, len(sections), (ctypes.c_int32 * 4)(*sections), T, H, G, D, (ctypes.c_int64 * 8)(*s), out)
    return tuple(out)


def test_shapes_with_several_tokens_a_workgroup():
    from test_gpu_rotary_axes_kernels import SEVERAL
    grains, tokens = set(), set()
    for (T, H, G, D, sections), (halves, own, each) in SEVERAL.items():
        for norm, has_bias in ((0, 0), (1, 0), (2, 1)):
            for pairing, grain in ((HALVES, halves), (NEIGHBOURS, 0), (AXIS_HALVES, own)):
                assert choice(norm, has_bias, pairing, T, H, G, D, sections) == (grain, 0, each, H + G)
                grains.add(grain)
        tokens.add(each)
    assert grains == {0, 1, 2, 4, 8} and {2, 4, 5, 6, 8} <= tokens
    assert choice(2, 1, AXIS_HALVES, 7257, 20, 4, 96, (4, 10, 10)) == (2, 0, 5, 24)


def test_heads_far_apart():
    from test_gpu_rotary_axes import PAIRINGS
    from test_gpu_rotary_axes_kernels import APART, FAR
    for (sections, pairing), grain in FAR.items():
        for norm, has_bias in ((0, 0), (1, 1), (2, 1)):
            for which in range(4):
                strides = [192, 64] * 4
                strides[2 * which:2 * which + 2] = 128, APART
                H, G = (3, 1) if which < 2 else (1, 3)
                assert choice(norm, has_bias, PAIRINGS.index(pairing), 3, H, G, 64, sections, strides)[:2] == (grain, 1)
    assert set(FAR.values()) == {0, 1, 2, 4, 8}
    assert choice(0, 0, HALVES, 2, 2, 0, 64, (8, 24), [64, 2**30 - 128] * 2 + [0] * 4)[1] == 0
    assert choice(0, 0, HALVES, 2, 2, 0, 64, (8, 24), [64, 2**30 - 64] * 2 + [0] * 4)[1] == 1


def test_few_tokens_are_dealt_by_heads():
    assert choice(0, 0, HALVES, 1, 32, 8, 128, (64,))[2:] == (1, 14)
    assert choice(1, 0, NEIGHBOURS, 700, 100, 10, 128, (64,))[2:] == (1, 55)
    assert choice(0, 0, HALVES, 768, 32, 8, 128, (64,))[2:] == (1, 40)
