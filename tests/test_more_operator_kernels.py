"""The kernels of rotary positions of several axes, norms, attention in a window and behind a prefix: which one a call reaches, and that none spills
registers."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2406_02540_amd import binding, build


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)


def window_choice(lq, lk, H, G, left, right, sinks, causal, more=0):
    out = (ctypes.c_int * 2)()
    binding.lib().vq_internal_attention_window_choice(len(lq), sum(lq) + more, sum(lk), H, G, int(causal), left, right, sinks, out)
    return out[0], out[1] > 0


def prefix_choice(lq, lk, P, H, G, D, more=0):
    out = (ctypes.c_int * 4)()
    binding.lib().vq_internal_attention_prefix_choice(len(lq), sum(lq) + more, P, sum(lk), H, G, D, out)
    return bool(out[0]), out[1], out[2] > 0, out[3] > 0


def test_every_kernel_of_the_window_is_reached_by_the_gpu_tests():
    pytest.importorskip("torch")
    from test_gpu_attention_more_kernels import WINDOW
    for name, (kernel, divided, lq, lk, H, G, left, right, sinks, causal) in WINDOW.items():
        assert len(lq) == len(lk), name
        for more in (0, 5):
            assert window_choice(lq, lk, H, G, left, right, sinks, causal, more) == (kernel, divided), name
    assert {(c[0], c[1]) for c in WINDOW.values()} == {(0, False), (0, True), (1, False), (1, True), (2, False)}


def test_every_kernel_behind_a_prefix_is_reached_by_the_gpu_tests():
    pytest.importorskip("torch")
    from test_gpu_attention_more_kernels import DIMS, PREFIX
    for name, (*want, lq, lk, P, H, G) in PREFIX.items():
        assert len(lq) == len(lk), name
        for D in DIMS:
            for more in (0, 5):
                assert prefix_choice(lq, lk, P, H, G, D, more) == tuple(want), (name, D)
    assert {(c[0], c[1], c[2]) for c in PREFIX.values()} == {(False, 0, False), (False, 0, True), (False, 1, False), (False, 1, True), (True, 1, False),
                                                             (True, 1, True), (True, 0, False), (True, 0, True)}
    assert {next(i for i, most in enumerate((64, 80, 96, 128)) if d <= most) for d in DIMS} == {0, 1, 2, 3}


@pytest.mark.parametrize("source", ["vq_rotary_axes.hip", "vq_attention_window.hip", "vq_attention_prefix.hip"])
def test_kernels_do_not_spill(source):
    if not os.path.exists(build.hipcc()):
        pytest.skip("no hipcc")
    out = subprocess.run([build.hipcc(), *build.HIPCC_FLAGS, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                          "--cuda-device-only", "-c", os.path.join(build.CSRC, source), "-o", os.devnull,
                          "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", out.stderr)
    scratch = [int(b) for b in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", out.stderr)]
    assert len(names) == len(scratch) > 0
    assert {n: b for n, b in zip(names, scratch) if b} == {}
