"""CPU checks of the ragged-batch calls and of the norms of queries and keys: the
binding's structures against the header, refusals in Python (before any pointer leaves
it) and at the C entry (under sanitizers, against launch stubs), the reference formulas
the GPU tests compare with, and the generated code."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2608_06838_amd as sf
from paper_2608_06838_amd import _lib

import _serve_ref as ref
from test_asm_stores import in_memory, overlapping_stores

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_06838_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def test_structures_match_the_header(tmp_path):
    """Sizes and offsets of the binding's structures are those a C compiler gives."""
    pairs = [("sf_ragged", _lib.SfRagged), ("sf_gdn_ragged_shape", _lib.SfGdnRaggedShape),
             ("sf_conv_ragged_shape", _lib.SfConvRaggedShape), ("sf_qk_shape", _lib.SfQkShape)]
    lines = []
    for c, py in pairs:
        lines.append(f'printf("%zu\\n", sizeof({c}));')
        lines += [f'printf("%zu\\n", offsetof({c}, {n}));' for n, _ in py._fields_]
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include "stateflow.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(tmp_path / "t")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "t")], capture_output=True, text=True).stdout.split()]
    want = []
    for _, py in pairs:
        want.append(ctypes.sizeof(py))
        want += [getattr(py, n).offset for n, _ in py._fields_]
    assert got == want
    text = open(os.path.join(ROOT, "include", "stateflow.h")).read()
    for name, kid in _lib.KERNELS.items():
        assert re.search(rf"SF_K_{name.upper()} = {kid}\b", text), name
    assert _lib.SF_NORM_RMS == 2 and "SF_NORM_RMS = 2" in text


def gdn_args(T=6, Hk=2, Hv=4, Dk=64, Dv=64, n=3):
    q, k, v = torch.randn(T, Hk, Dk), torch.randn(T, Hk, Dk), torch.randn(T, Hv, Dv)
    return dict(q=q, k=k, v=v, g=torch.zeros(T, Hv), beta=torch.zeros(T, Hv), state=torch.zeros(n, Hv, Dk, Dv),
                cu_seqlens=torch.zeros(n + 1, dtype=torch.int32), slots=torch.zeros(n, dtype=torch.int32))


@pytest.mark.parametrize("change", [
    dict(), dict(q=torch.randn(6, 2, 64).half()), dict(k=torch.randn(6, 2, 32)), dict(k=torch.randn(6, 2, 64).bfloat16()),
    dict(q=torch.randn(6, 128)), dict(v=torch.randn(5, 4, 64)), dict(g=torch.zeros(6, 4).double()),
    dict(beta=torch.zeros(6, 2)), dict(beta=torch.zeros(4, 6).t()), dict(state=torch.zeros(3, 4, 64, 32)),
    dict(state=torch.zeros(3, 4, 64, 64).bfloat16()), dict(state=torch.zeros(3, 4, 64, 64).transpose(2, 3)),
    dict(cu_seqlens=torch.zeros(4, dtype=torch.int64)), dict(cu_seqlens=torch.zeros(0, dtype=torch.int32)),
    dict(slots=torch.zeros(2, dtype=torch.int32)), dict(slots=torch.zeros(3)), dict(fresh=torch.zeros(3)),
    dict(fresh=torch.zeros(4, dtype=torch.bool)), dict(out=(torch.zeros(6, 4, 32), None)),
    dict(q=torch.randn(6, 64, 2).transpose(1, 2), k=torch.randn(6, 64, 2).transpose(1, 2))])
def test_gdn_refusals(change):
    """Wrong shapes and types; and, with all of them right, host memory."""
    with pytest.raises((ValueError, TypeError)) as e:
        sf.gdn_ragged_fwd(**{**gdn_args(), **change})
    assert change or "must be on" in str(e.value)


@pytest.mark.parametrize("change", [
    dict(), dict(x=torch.randn(6, 64).half()), dict(x=torch.randn(64, 6).t()), dict(x=torch.randn(1, 6, 64)),
    dict(w=torch.randn(32, 4)), dict(w=torch.randn(64, 4).bfloat16()), dict(w=torch.randn(4, 64).t()),
    dict(tails=None), dict(tails=torch.zeros(3, 2, 64)), dict(tails=torch.zeros(3, 64, 3).transpose(1, 2)),
    dict(act="relu"), dict(out=torch.zeros(6, 32)), dict(cu_seqlens=torch.zeros(2, 2, dtype=torch.int32))])
def test_conv_refusals(change):
    args = dict(x=torch.randn(6, 64), w=torch.randn(64, 4), tails=torch.zeros(3, 3, 64),
                cu_seqlens=torch.zeros(4, dtype=torch.int32), slots=torch.zeros(3, dtype=torch.int32))
    with pytest.raises((ValueError, TypeError)) as e:
        sf.conv_ragged_fwd(**{**args, **change})
    assert change or "must be on" in str(e.value)


@pytest.mark.parametrize("change", [
    dict(), dict(norm="layer"), dict(q=torch.randn(1, 3, 4, 64).half()), dict(k=torch.randn(1, 3, 2, 32)),
    dict(k=torch.randn(1, 4, 2, 64)), dict(k=torch.randn(1, 3, 2, 64).bfloat16()), dict(q=torch.randn(3, 4, 64)),
    dict(q_weight=torch.randn(32)), dict(k_weight=torch.randn(64).double()), dict(inv_freq=torch.randn(16)),
    dict(inv_freq=torch.randn(16).double(), pos=torch.zeros(1, 3)), dict(pos=torch.zeros(3, dtype=torch.int64)),
    dict(q=torch.randn(1, 3, 64, 4).transpose(2, 3))])
def test_qk_refusals(change):
    args = {**dict(q=torch.randn(1, 3, 4, 64), k=torch.randn(1, 3, 2, 64)), **change}
    for out in (None, (torch.zeros(1, 3, 4, 64), torch.zeros(1, 3, 2, 32))):
        with pytest.raises((ValueError, TypeError)) as e:
            sf.qk_norm_fwd(**args, out=out)
        assert change or out or "must be on" in str(e.value)
    with pytest.raises((ValueError, TypeError)):
        sf.qk_norm_bwd(args.pop("q"), args.pop("k"), torch.zeros(1, 3, 4, 64), torch.zeros(1, 3, 2, 64), **args)


def test_reference_gradients():
    """The formulas the GPU gradients are compared with, against 64-bit autograd."""
    torch.manual_seed(0)
    for norm, inter, R in (("l2", False, 32), ("rms", True, 16), ("none", False, 32), ("rms", False, 0)):
        q, k = (torch.randn(2, 3, h, 32, dtype=torch.float64, requires_grad=True) for h in (2, 1))
        dyq, dyk = torch.randn_like(q), torch.randn_like(k)
        wq, wk = (torch.randn(32, dtype=torch.float64, requires_grad=True) for _ in range(2))
        f = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / max(R, 1)) if R else None
        kw = dict(norm=norm, q_scale=0.4, inv_freq=f, pos0=7, interleaved=inter, q_weight=wq, k_weight=wk)

        def forward(x, w, s):
            c = {"none": 0.0, "l2": 1.0, "rms": 1 / 32}[norm]
            y = w * (x if norm == "none" else x / (c * (x * x).sum(-1, keepdim=True) + 1e-6).sqrt())
            if R:
                ang = ((7 + torch.arange(3.0, dtype=torch.float64))[:, None] * f)[None, :, None]
                a, b = (y[..., 0:R:2], y[..., 1:R:2]) if inter else (y[..., :R // 2], y[..., R // 2:R])
                a, b = a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()
                y = torch.cat([torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1), y[..., R:]], -1)
            return s * y

        yq, yk = forward(q, wq, 0.4), forward(k, wk, 1.0)
        for got, want in zip(ref.qk(q, k, **kw), (yq, yk)):
            np.testing.assert_allclose(got, want.detach().numpy(), atol=1e-12)
        ((yq * dyq).sum() + (yk * dyk).sum()).backward()
        (gq, gwq, _), (gk, gwk, _) = ref.qk(q, k, **kw, dyq=dyq, dyk=dyk)
        np.testing.assert_allclose(gq, q.grad.numpy(), atol=1e-12)
        np.testing.assert_allclose(gk, k.grad.numpy(), atol=1e-12)
        np.testing.assert_allclose(gwq, wq.grad.numpy(), atol=1e-11)
        np.testing.assert_allclose(gwk, wk.grad.numpy(), atol=1e-11)


def test_reference_recurrence_and_convolution():
    """The ragged references against the oracle, sequence by sequence."""
    import oracle
    from oracle import gdn as gdo
    rng = np.random.RandomState(0)
    lens, H, D = [3, 0, 5], 2, 4
    cu = np.cumsum([0] + lens)
    q, k, v = (torch.tensor(rng.randn(8, H, D)) for _ in range(3))
    g, beta = -torch.tensor(rng.rand(8, H)), torch.tensor(rng.rand(8, H))
    S = torch.tensor(rng.randn(4, H, D, D))
    o, written, new = ref.gdn(q, k, v, g, beta, S, cu, [2, 0, 1], [0, 1, 1])
    x, w, tails = torch.tensor(rng.randn(8, 6)), torch.tensor(rng.randn(6, 3)), torch.tensor(rng.randn(4, 2, 6))
    y, _, nt = ref.conv(x, w, tails, cu, [2, 0, 1], [0, 1, 1])
    for b, e, slot, fresh in ((0, 3, 2, 0), (3, 8, 1, 1)):
        wo, wS = gdo.forward(*[t[None, b:e] for t in (q, k, v, g, beta)], None if fresh else S[None, slot])
        np.testing.assert_allclose(o[b:e], wo[0], atol=1e-12)
        np.testing.assert_allclose(new[slot], wS[0], atol=1e-12)
        wy, wt = oracle.conv_forward(x[None, b:e], w, None if fresh else tails[None, slot])
        np.testing.assert_allclose(y[b:e], wy[0], atol=1e-12)
        np.testing.assert_allclose(nt[slot], wt[0], atol=1e-12)
    assert written.all() and np.array_equal(new[[0, 3]], S[[0, 3]]) and np.array_equal(nt[[0, 3]], tails[[0, 3]])


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_entry_points_under_sanitizers(tmp_path):
    exe = str(tmp_path / "serve_checks")
    san = os.path.join(ROOT, "tests", "sanitize")
    # sanitizers on the host pass only
    cmd = [HIPCC, "-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fno-omit-frame-pointer",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", *FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-I", san, os.path.join(CSRC, "sf_abi.hip"), os.path.join(CSRC, "sf_abi_serve.hip"),
           *(os.path.join(san, f) for f in ("launch_stubs.cpp", "serve_stubs.cpp", "serve_checks.cpp")), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120, env={
        **os.environ, "ASAN_OPTIONS": "detect_leaks=0:verify_asan_link_order=0", "UBSAN_OPTIONS": "print_stacktrace=1"})
    assert res.returncode == 0 and "serve checks passed" in res.stdout, res.stdout + res.stderr


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
@pytest.mark.parametrize("src,most", [("sf_ragged.hip", 20), ("sf_qk.hip", 41), ("sf_ragged_chunk.hip", 4)])
def test_generated_code(src, most, tmp_path):
    """No store over its own address, no scratch memory, nothing read before it is written."""
    out = str(tmp_path / "k.s")
    res = subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "--cuda-device-only", "-S",
                          "-Wuninitialized", "-Wconditional-uninitialized", "-Wsometimes-uninitialized", *FLAGS, "-I",
                          os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(CSRC, src), "-o", out],
                         check=True, capture_output=True, text=True)
    assert "uninitialized" not in res.stderr, res.stderr
    asm = open(out).read()
    n, bad = overlapping_stores(asm)
    kernels, kept = in_memory(asm)
    assert kernels >= most and not kept, kept[:3]
    assert n > 50 and not bad, bad[:3]
