"""The host side of attention (refusals, choices of kernels and divisions, workspaces) once more against a build with
UndefinedBehaviorSanitizer in host code.  CPU only."""
import os
import subprocess

import pytest

from test_sanitizers import ROOT, _child_env, _run_pytest

SAN = ["-fsanitize=undefined", "-fno-sanitize-recover=undefined"]
SOURCES = ["vq_api.hip", "vq_attention.hip", "vq_attention_window.hip", "vq_attention_prefix.hip"]


def test_attention_host_side_under_sanitizers(tmp_path):
    from paper_2406_02540_amd import build as hb
    hipcc = hb.hipcc()
    probe = subprocess.run([hipcc, "-print-file-name=libclang_rt.ubsan_standalone-x86_64.so"], capture_output=True, text=True)
    runtime = os.path.realpath(probe.stdout.strip()) if probe.returncode == 0 else ""
    if not os.path.isabs(runtime) or not os.path.exists(runtime):
        pytest.skip("hipcc's clang has no UndefinedBehaviorSanitizer runtime here")
    others = [os.path.join(hb.CSRC, s.replace(".hip", ".o")) for s in hb.SOURCES if s not in SOURCES]
    if not all(os.path.exists(o) for o in others):
        hb.build(verbose=False)
    host_san = [f for flag in SAN for f in ("-Xarch_host", flag)]
    flags = [f for f in hb.HIPCC_FLAGS if f != "-O3"]
    objs = [str(tmp_path / s.replace(".hip", ".o")) for s in SOURCES]
    procs = [subprocess.Popen([hipcc, *flags, "-O1", "-g", *host_san, "-I", os.path.join(ROOT, "include"), "-I", hb.CSRC, "-c", os.path.join(hb.CSRC, s), "-o", o],
                              stderr=subprocess.DEVNULL) for s, o in zip(SOURCES, objs)]
    assert [p.wait() for p in procs] == [0] * len(procs)
    lib = str(tmp_path / "libvidiq_san.so")
    subprocess.check_call([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *host_san, "-shared-libsan", *objs, *others, "-o", lib], stderr=subprocess.DEVNULL)
    _run_pytest(["tests/test_attention_division.py", "tests/test_more_operators_host.py", "tests/test_operators_host.py"], _child_env(runtime, {"VQ_LIBVIDIQ_PATH": lib}))
