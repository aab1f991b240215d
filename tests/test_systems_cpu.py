"""Chunk systems of the ragged delta rule: how they are numbered, what workspace they
take, and the length a call without max_len assumes."""
import os
import subprocess

import pytest
import torch

import paper_2608_06838_amd as sf

from test_serve_cpu import CSRC, FLAGS, HIPCC, ROOT


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_numbering_under_sanitizers(tmp_path):
    exe = str(tmp_path / "system_checks")
    san = os.path.join(ROOT, "tests", "sanitize")
    cmd = [HIPCC, "-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fno-omit-frame-pointer",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", *FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-I", san, os.path.join(CSRC, "sf_abi.hip"), os.path.join(CSRC, "sf_abi_serve.hip"),
           *(os.path.join(san, f) for f in ("launch_stubs.cpp", "serve_stubs.cpp", "system_checks.cpp")), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120, env={
        **os.environ, "ASAN_OPTIONS": "detect_leaks=0:verify_asan_link_order=0", "UBSAN_OPTIONS": "print_stacktrace=1"})
    assert res.returncode == 0 and "system checks passed" in res.stdout, (res.stdout + res.stderr)[-3000:]


@pytest.mark.parametrize("T,N,want", [(256, 256, 1), (2111, 64, 2048), (1000, 1024, 1000), (0, 3, 0), (5, 1, 5)])
def test_length_without_a_hint(T, N, want):
    """One token each but for one sequence; fewer tokens than sequences say nothing: any
    one of them may have all."""
    state, cu = torch.zeros(N, 1, 64, 64), torch.zeros(N + 1, dtype=torch.int32)
    assert sf._ragged(T, state, cu, None, None, None).max_len == want
    assert sf._ragged(T, state, cu, None, None, 7).max_len == 7
