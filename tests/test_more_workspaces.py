"""Workspace sizes of attention in a window and behind a prefix asked for from Python: what the calls themselves refuse has none."""
import os

import pytest

pytest.importorskip("torch")

from paper_2406_02540_amd import binding, build  # noqa: E402
import paper_2406_02540_amd as vq  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)


WINDOW = (2, 2, 80000, 8, 2, 128, False, 30000, 0, 4)
PREFIX = (40, 40, 20000, 4000, 8, 2, 128)


@pytest.mark.parametrize("at", [i for i in range(len(WINDOW)) if i != 6])
def test_numbers_of_a_window_that_do_not_fit(at):
    need = vq.vq_attention_window_workspace_bytes(*WINDOW)
    assert need > 0
    for more in (2**32, -2**32, 2**40):
        sizes = list(WINDOW)
        sizes[at] += more
        assert vq.vq_attention_window_workspace_bytes(*sizes) == 0


@pytest.mark.parametrize("at", range(len(PREFIX)))
def test_numbers_of_a_prefix_that_do_not_fit(at):
    assert vq.vq_attention_prefix_workspace_bytes(*PREFIX) > 0
    for more in (2**32, -2**32, 2**40):
        sizes = list(PREFIX)
        sizes[at] += more
        assert vq.vq_attention_prefix_workspace_bytes(*sizes) == 0


def test_windows_that_are_no_whole_numbers():
    # (as the call has it)
    for at, value in ((7, 30000.5), (7, "far"), (8, 1.0), (9, 4.5), (9, None)):
        sizes = list(WINDOW)
        sizes[at] = value
        with pytest.raises(TypeError):
            vq.vq_attention_window_workspace_bytes(*sizes)
    assert vq.vq_attention_window_workspace_bytes(*WINDOW[:7], None, None, 0) == vq.vq_attention_window_workspace_bytes(*WINDOW[:7], -1, -1, 0) > 0
