"""The kernels of microscaled layers, rotary positions and attention: which one a product reaches, and that none spills registers."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2406_02540_amd import binding, build

CUS = 256   # of an MI355X


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)


def choice(M, N, K):
    """(tokens, channels, whether the wavefronts divide K) of the tile that a product takes."""
    out = (ctypes.c_int * 3)()
    binding.lib().vq_internal_mx4_choice(M, N, K, CUS, out)
    return tuple(out)


def test_every_tile_is_reached_by_the_gpu_tests():
    pytest.importorskip("torch")
    from test_gpu_mx4 import LARGE, SIZES
    assert {choice(*s) for s in SIZES + LARGE} == {(256, 256, 0), (128, 128, 0), (64, 128, 0), (32, 32, 1), (48, 48, 1), (32, 64, 1)}


def test_choice_of_large_and_ragged_rows():
    assert choice(32768, 4608, 1152) == (256, 256, 0)
    assert choice(32768, 4607, 1152)[0] < 256          # rows that are no whole pieces: not the largest tile
    for M, N in ((700_000_000, 8), (1, 700_000_000), (1_000_000_000, 32)):
        t, c, divide = choice(M, N, 32)
        assert not divide or -(-M // t) * -(-N // c) * 512 < 2 ** 32


@pytest.mark.parametrize("source", ["vq_mx4_quantize.hip", "vq_mx4_gemm.hip", "vq_mx4_gemm_split.hip", "vq_rotary.hip", "vq_attention.hip",
                                    "vq_attention_tiles.hip"])
def test_kernels_do_not_spill(source):
    if not os.path.exists(build.hipcc()):
        pytest.skip("no hipcc")
    out = subprocess.run([build.hipcc(), *build.HIPCC_FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                          "--cuda-device-only", "-c", os.path.join(build.CSRC, source), "-o", os.devnull,
                          "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", out.stderr)
    scratch = [int(b) for b in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", out.stderr)]
    assert len(names) == len(scratch) > 0
    assert {n: b for n, b in zip(names, scratch) if b} == {}


def test_wide_rows_reach_the_stores_of_any_row():
    pytest.importorskip("torch")
    from test_gpu_mx4_wide import WIDE
    assert all(N >= 1 << 21 and not choice(M, N, K)[2] for M, N, K in WIDE)
    assert any(N % 8 == 0 for _, N, _ in WIDE) and any(2 * N * min(M, choice(M, N, K)[0]) >= 1 << 31 for M, N, K in WIDE)


def test_every_attention_kernel_is_reached_by_the_gpu_tests():
    pytest.importorskip("torch")
    from test_gpu_attention_kernels import BAD_SHAPES, CASES, DIMS

    def attention_choice(*sizes):
        out = (ctypes.c_int * 2)()
        binding.lib().vq_internal_attention_choice(*sizes, out)
        return out[0], out[1] > 0

    for name, (kernel, divided, lq, lk, H, G) in CASES.items():
        assert attention_choice(len(lq), sum(lq) + 5, sum(lk), H, G) == attention_choice(len(lq), sum(lq), sum(lk), H, G) == (kernel, divided), name
        # its rows and its keys in several turns
        assert max(lq) * H // G > (128 if kernel == 0 else 32) and max(lk) > 64 or name == "frames", name
    assert {(c[0], c[1]) for c in CASES.values()} == {(0, False), (0, True), (1, False), (1, True), (2, False)}
    assert {next(i for i, most in enumerate((64, 80, 96, 128)) if d <= most) for d in DIMS} == {0, 1, 2, 3}
    assert [attention_choice(4, 100, Tk, H, G) for H, G, Tk, _, _ in BAD_SHAPES] == [s[3:] for s in BAD_SHAPES]
