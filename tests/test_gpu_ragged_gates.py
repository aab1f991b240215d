"""Strong gates beside weak ones inside one chunk of the ragged delta rule: resets (g =
-inf) of packed documents, and finite gates down to -50, each with weak ones behind it in
the sequence's last chunk, against plain 64-bit runs on both sides of max_len.

What is allowed: test_gpu_ragged.py derives 1e-5 of the RMS for the largest of 10^6
elements of fp32 arithmetic; twice that here.  A decay formed as the difference of two
fp32 running sums b would be off by ulp(b), whatever its own size: 4 resets leave b near
600, 6e-5, and the largest element of state or output near 1e-4.
"""
import numpy as np
import pytest
import torch

from test_gpu_ragged import gdn_inputs, run_gdn

pytestmark = pytest.mark.gpu
DELTA = 2e-5
INF = float("inf")


def resets(n, every, count):
    at = np.zeros(n, bool)
    at[every // 2:every * count:every] = True
    return at, np.full(n, -INF)


def strong(n, count, mean, seed=0):
    at = np.arange(n) < count
    return at, mean * (0.8 + 0.4 * np.random.RandomState(seed).rand(n))


# where in the sequence's last chunk the gates are strong, and their values
GATES = {"3 resets": resets(64, 8, 3), "8 resets": resets(64, 6, 8), "40 resets": resets(64, 1, 40),
         "32 at -5": strong(64, 32, -5.0), "32 at -20": strong(64, 32, -20.0), "50 at -50": strong(64, 50, -50.0)}


@pytest.mark.parametrize("name", list(GATES))
@pytest.mark.parametrize("Hk,Hv,Dk,Dv", [(1, 2, 128, 128), (1, 1, 64, 64)])
def test_strong_gates_before_weak_ones(name, Hk, Hv, Dk, Dv):
    lens = [64, 128 + 61, 100]
    cu = np.cumsum([0] + lens)
    print(f"[gdn ragged] {name}, heads of {Dk} x {Dv}", flush=True)
    for max_len in (1, max(lens)):
        args = gdn_inputs(int(cu[-1]), Hk, Hv, Dk, Dv, len(lens), seed=31)
        at, val = GATES[name]
        for b, e in zip(cu, cu[1:]):
            c0 = b + (e - b - 1) // 64 * 64  # the last chunk; at least 8 weak gates stay behind the strong ones
            m = at[:e - c0].copy()
            m[e - c0 - 8:] = False
            rows = torch.tensor(c0 + np.flatnonzero(m), device=args[3].device)
            args[3][rows] = torch.tensor(val[:e - c0][m], dtype=torch.float32, device=args[3].device)[:, None]
        run_gdn(args, cu, max_len=max_len, delta=DELTA)
