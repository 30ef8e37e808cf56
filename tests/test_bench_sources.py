"""The hash by which bench.py takes a summary of counters: of the int8 kernels' sources, and of nothing else."""
import importlib.util
import json
import os
import re
import shutil

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join("paper_2406_02540_amd", "csrc")


@pytest.fixture
def bench(tmp_path, monkeypatch):
    """bench.py on a copy of the sources."""
    spec = importlib.util.spec_from_file_location("bench_under_test", os.path.join(ROOT, "bench.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    (tmp_path / CSRC).mkdir(parents=True)
    for f in os.listdir(os.path.join(ROOT, CSRC)):
        if f.endswith((".hip", ".h")):
            shutil.copy(os.path.join(ROOT, CSRC, f), tmp_path / CSRC)
    monkeypatch.setattr(module, "ROOT", str(tmp_path))
    return module


def _sources(names):
    """The files and what they include of csrc, over and over."""
    found, rest = set(), list(names)
    while rest:
        f = rest.pop()
        if f in found or not os.path.exists(os.path.join(ROOT, CSRC, f)):
            continue
        found.add(f)
        rest += re.findall(r'#include "([^"]+)"', open(os.path.join(ROOT, CSRC, f)).read())
    return found


def test_hash_is_of_the_int8_kernels(bench, tmp_path):
    from paper_2406_02540_amd import build
    others = ("vq_api.hip", "vq_mx4", "vq_rotary", "vq_attention")
    kernels = _sources(f for f in build.SOURCES if not f.startswith(others)) - {"vq_internal.h"}     # (declarations)
    first = bench.csrc_hash()
    for f in sorted(os.listdir(tmp_path / CSRC)):
        path = tmp_path / CSRC / f
        text = path.read_bytes()
        path.write_bytes(text + b"\n// another line\n")
        assert (bench.csrc_hash() != first) == (f in kernels), f
        path.write_bytes(text)
    (tmp_path / CSRC / "vq_attention_more.hip").write_text("// another operator\n")
    assert bench.csrc_hash() == first


def test_counters_name_their_sources():
    for workload in ("video", "video_w4", "image"):
        t = json.load(open(os.path.join(ROOT, "profiles", f"gemm_counters_{workload}.json")))
        assert re.fullmatch("[0-9a-f]{16}", t["csrc_sha256"]) and t["layers"] and os.path.exists(os.path.join(ROOT, t["source"]))
