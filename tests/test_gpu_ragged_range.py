"""Ragged delta rule near the ends of fp32's range: output and state are linear in value
and state together, so a run with both times 2^110 or 2^-90 (exact) is the plain run
times that.  Tolerances as in test_gpu_ragged.py."""
import numpy as np
import pytest
import torch

import paper_2608_06838_amd as sf

import _serve_ref as ref
from _serve_ref import close
from test_gpu_ragged import DELTA, gdn_inputs, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("power", [110, -90])
@pytest.mark.parametrize("gate", [-3.0, 0.3])
def test_large_and_small_values(io, power, gate):
    """Decay that leaves 1e-9 behind within seven tokens; growth of 1e3 within 24."""
    print(f"[gdn ragged] {io} values times 2^{power}, gates near {gate}", flush=True)
    lens = [24, 1, 40, 7] if gate < 0 else [24, 1, 20, 7]
    cu = np.cumsum([0] + lens)
    for max_len in (1, max(lens)):
        args = gdn_inputs(int(cu[-1]), 1, 2, 64, 64, len(lens), io, seed=91)
        args[3] = gate * (0.5 + torch.rand(args[3].shape, generator=torch.Generator().manual_seed(1)).to(args[3].device))
        want_o, _, want_S = ref.gdn(*args, cu, None)
        args[2], args[5] = args[2] * 2.0 ** power, args[5] * 2.0 ** power
        o = sf.gdn_ragged_fwd(*args, i32(cu), max_len=max_len)
        torch.cuda.synchronize()
        close("o", o, want_o * 2.0 ** power, DELTA)
        close("state", args[5], want_S * 2.0 ** power, DELTA)
