"""Outputs and gradients of the norms as slices of one [B, H, L, D] buffer, seen as
[B, L, H, D]: batch by batch the queries' part and the keys' lie in turn."""
import pytest
import torch

import paper_2608_06838_amd as sf

from test_gpu_qk import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_heads_outermost_in_one_buffer(io):
    B, L, Hq, Hk, D = 3, 19, 4, 2, 64
    print(f"[qk] {io} heads outermost, one buffer", flush=True)
    t, kw = make(B, L, Hq, Hk, D, io, seed=61, R=32)
    y, d = (torch.full((B, Hq + Hk + 1, L, D), 7.0, dtype=t[0].dtype, device=t[0].device) for _ in range(2))
    views = lambda b: (b[:, :Hq].transpose(1, 2), b[:, Hq:Hq + Hk].transpose(1, 2))  # noqa: E731
    ws = torch.empty(sf.qk_norm_bwd_workspace_bytes(*t), dtype=torch.uint8, device=t[0].device)
    dw = [torch.empty(D, device=t[0].device) for _ in range(2)]
    check(t, dict(kw, norm="rms"), out_f=views(y), out_b=(*views(d), *dw, ws))
    assert bool((y[:, Hq + Hk] == 7).all()) and bool((d[:, Hq + Hk] == 7).all())
