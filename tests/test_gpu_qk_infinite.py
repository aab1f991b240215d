"""Norms of queries and keys where values are infinite or their products overflow:
without a norm the gradient does not depend on x.  Tolerances as in test_gpu_qk.py."""
import pytest
import torch

import paper_2608_06838_amd as sf

import _serve_ref as ref
from _serve_ref import close
from test_gpu_qk import DELTA, make

pytestmark = pytest.mark.gpu
INF = float("inf")


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
