"""The rotation's sines and cosines, seen by turning unit vectors in fp32 without a norm:
each is held relative to its own size.

sin and cos of a float are off by at most 4 units in the last place, 4 2^-23; the angle's
part below a float is added in first order, and its own rounding and the angle's 64-bit
forming (650 turns 2^-52 2 pi = 1e-12) stay below 1e-8 of values above 1e-4.  Allowed:
2^-21 + 1e-8.  An angle rounded to a float would be off by up to pi 2^-25, 1e-3 of a
cosine of 1e-4.
"""
import numpy as np
import pytest
import torch

import paper_2608_06838_amd as sf

import _serve_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("back", [False, True])
def test_sines_and_cosines_to_their_own_size(inter, back):
    L, D = 4096, 64
    n = D // 2
    print(f"[qk] angles interleaved={inter} backward={back}", flush=True)
    inv_freq = 10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)
    first = slice(0, D, 2) if inter else slice(0, n)
    second = slice(1, D, 2) if inter else slice(n, D)
    x = torch.zeros(1, L, 1, D)
    x[..., first] = 1.0
    x = x.to(DEV)
    kw = dict(norm="none", inv_freq=inv_freq.to(DEV), interleaved=inter)
    if back:
        y = sf.qk_norm_bwd(x, x, x, x, **kw)[0]
    else:
        y = sf.qk_norm_fwd(x, x, **kw)[0]
    torch.cuda.synchronize()
    y = ref.f64(y)[0, :, 0]
    ang = np.arange(L, dtype=np.float64)[:, None] * inv_freq.numpy() * (-1 if back else 1)
    for got, want in ((y[:, first], np.cos(ang)), (y[:, second], np.sin(ang))):
        use = np.abs(want) > 1e-4
        off = np.abs(got - want)[use] / np.abs(want[use])
        print(f"  {use.sum()} values, worst {off.max() * 2 ** 23:.2f} units", flush=True)
        assert off.max() <= 2.0 ** -21 + 1e-8
