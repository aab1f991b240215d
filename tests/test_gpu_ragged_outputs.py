"""The bf16 outputs of the ragged delta rule in chunks are the 64-bit values rounded once.

An output whose error before the rounding is d lands on the wrong neighbour with
probability d / h, h the bf16 step there.  fp32 arithmetic with every product above 2^-24
kept leaves about 8 2^-24 of the RMS (sums of 64 to 128 terms in three products one
behind the other).  Among outputs of at least half the RMS, h is 2^-8 RMS or more, and
on average over a normal distribution 1 / h is below 170 / RMS: a share of
0.8 8 2^-24 170 = 6.5e-5.  Allowed: 1e-4.  Operands of 17 bits (pairs) would show 2e-4.
"""
import numpy as np
import pytest
import torch

import paper_2608_06838_amd as sf

import _serve_ref as ref
from test_gpu_ragged import gdn_inputs, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,lens,Hk,Hv,Dk,Dv", [
    ("one prompt, single column tiles", [2500], 2, 4, 128, 128),
    ("many prompts, pairs of tiles", [192, 250] * 8, 4, 4, 128, 128),
    ("narrow keys", [1500, 900], 2, 4, 64, 128)])
def test_outputs_are_rounded_once(name, lens, Hk, Hv, Dk, Dv):
    cu = np.cumsum([0] + lens)
    print(f"[gdn ragged] {name}", flush=True)
    args = gdn_inputs(int(cu[-1]), Hk, Hv, Dk, Dv, len(lens), seed=41)
    want, _, _ = ref.gdn(*args, cu, None)
    o = sf.gdn_ragged_fwd(*args, i32(cu), max_len=max(lens))
    torch.cuda.synchronize()
    far = np.abs(want) >= 0.5 * np.sqrt(np.mean(want * want))
    step = 2.0 ** (np.floor(np.log2(np.abs(want[far]))) - 7)
    off = np.abs(ref.f64(o)[far] - want[far]) / step
    share = float(np.mean(off > 0.5 + 1e-9))
    print(f"  {far.sum()} outputs, share on the wrong side {share:.2e}, worst {off.max():.4f} of a step", flush=True)
    assert off.max() < 1
    assert share <= 1e-4
