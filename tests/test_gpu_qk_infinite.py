"""Norms of queries and keys where values are infinite or their products overflow:
channels behind the rotated ones pass through as they are, and without a norm the
gradient does not depend on x.  Tolerances as in test_gpu_qk.py."""
import numpy as np
import pytest
import torch

import paper_2608_06838_amd as sf

import _serve_ref as ref
from _serve_ref import close
from test_gpu_qk import DELTA, make

pytestmark = pytest.mark.gpu
INF = float("inf")


def same_places(name, X, R):
    """Infinities where the reference has them, everything else as ever."""
    x, R = ref.f64(X), R.copy()
    fine = np.isfinite(R)
    assert np.array_equal(x[~fine], R[~fine]), name
    x[~fine] = R[~fine] = 0
    close(name, torch.tensor(x).to(X.dtype), R, DELTA)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,R", [(128, 32), (96, 48), (32, 16)])
def test_channels_behind_the_rotation_pass_through(io, inter, D, R):
    print(f"[qk] {io} D={D} R={R} interleaved={inter}, infinite behind", flush=True)
    for weight in (True, False):
        t, kw = make(1, 5, 3, 2, D, io, seed=51, weight=weight, R=R)
        kw = dict(kw, norm="none", interleaved=inter)
        for x in t:
            x[0, 1, 0, R] = INF
            x[0, 2, 1, D - 1] = -INF
        yq, yk = sf.qk_norm_fwd(*t[:2], **kw)
        dq, dk, _, _ = sf.qk_norm_bwd(t[0].nan_to_num(0, 1, -1), t[1].nan_to_num(0, 1, -1), *t[2:], **kw)
        torch.cuda.synchronize()
        wq, wk = ref.qk(*t[:2], **kw)
        same_places("yq", yq, wq)
        same_places("yk", yk, wk)
        # without a norm the gradient is dy, turned back and weighted
        dy = ref.qk(*t[2:], norm="none", inv_freq=-kw["inv_freq"], pos=kw["pos"], interleaved=inter)
        w = [ref.f64(kw.get(n)) if weight else np.ones(D) for n in ("q_weight", "k_weight")]
        same_places("dq", dq, dy[0] * w[0])
        same_places("dk", dk, dy[1] * w[1])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("R", [0, 64])
def test_without_a_norm_the_gradient_ignores_x(io, R):
    """x infinite or NaN, and x and dy so large that their product overflows."""
    print(f"[qk] {io} R={R} no norm", flush=True)
    t, kw = make(1, 6, 2, 1, 64, io, seed=52, weight=False, R=R)
    kw = dict(kw, norm="none", q_scale=0.5)
    want = ref.qk(*t[:2], **kw, dyq=t[2], dyk=t[3])
    q, k = t[0].clone(), t[1].clone()
    q[0, 1, 0, 3] = INF
    q[0, 2, 1, 40] = float("nan")
    k[0, 3] = -INF
    dq, dk, _, _ = sf.qk_norm_bwd(q, k, *t[2:], **kw)
    torch.cuda.synchronize()
    close("dq", dq, want[0][0], DELTA)
    close("dk", dk, want[1][0], DELTA)
    big = [x * 2.0 ** 66 for x in t]  # exact
    dq, dk, _, _ = sf.qk_norm_bwd(*big, **kw)
    torch.cuda.synchronize()
    close("dq", dq, want[0][0] * 2.0 ** 66, DELTA)
    close("dk", dk, want[1][0] * 2.0 ** 66, DELTA)
