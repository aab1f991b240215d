"""The ragged delta rule where short and empty sequences outnumber the long ones, so that
the chunk systems are numbered by tokens alone: against plain 64-bit runs, with a workspace
full of NaN bytes.  Tolerances as in test_gpu_ragged.py."""
import numpy as np
import pytest
import torch

import paper_2608_06838_amd as sf

import _serve_ref as ref
from test_gpu_ragged import DELTA, gdn_inputs, i32, run_gdn
from _serve_ref import close

pytestmark = pytest.mark.gpu


def batches():
    rng = np.random.RandomState(9)
    yield "one prompt among single tokens", [1] * 150 + [333] + [1] * 100, 333
    yield "one prompt among empty sequences", [0] * 200 + [300] + [0] * 200, None
    lens = [1] * 200 + [13, 25, 64, 65, 128, 129, 24, 12, 26] + [0] * 60
    rng.shuffle(lens)
    yield "lengths at every line", [int(x) for x in lens], 129
    yield "long ones side by side", [25, 25, 65, 26, 0, 0, 129, 64] + [0] * 100, 129


@pytest.mark.parametrize("name,lens,max_len", list(batches()), ids=lambda x: x if isinstance(x, str) else "")
def test_many_short_sequences(name, lens, max_len):
    cu, T = ref.sequences(lens)
    print(f"[gdn ragged] {name}: {len(lens)} sequences, {T} tokens", flush=True)
    args = gdn_inputs(T, 1, 2, 64, 64, len(lens), seed=71)
    start = args[5].clone()
    run_gdn(args, cu, max_len=max_len)
    args[5].copy_(start)
    ws = torch.full((sf.gdn_ragged_workspace_bytes(*args, i32(cu), max_len=max_len),), 255, dtype=torch.uint8,
                    device=args[0].device)
    assert 0 < ws.numel() <= T // 13 * 2 * 37 * 1024 + 4 * (len(lens) + 2)
    o = sf.gdn_ragged_fwd(*args, i32(cu), max_len=max_len, out=(torch.empty_like(args[2]), ws))
    torch.cuda.synchronize()
    want_o, _, want_S = ref.gdn(*args[:5], start, cu, None)
    close("o", o, want_o, DELTA)
    close("state", args[5], want_S, DELTA)


def test_decreasing_bounds():
    """Bounds in any order: rows and slots that no sequence names keep their bits."""
    T, N = 400, 150
    rng = np.random.RandomState(3)
    print("[gdn ragged] bounds in any order", flush=True)
    args = gdn_inputs(T, 1, 2, 64, 64, N + 1, seed=72)
    for cu in (rng.randint(-50, T + 50, N + 1), np.sort(rng.randint(0, T + 1, N + 1))[::-1].copy()):
        at = np.clip(cu, 0, T)
        named = np.zeros(T, bool)
        for b, e in zip(at, at[1:]):
            named[b:e] = True
        S, o = args[5].clone(), torch.full(args[2].shape, 7.0, dtype=torch.bfloat16, device=args[0].device)
        ws = torch.zeros(sf.gdn_ragged_workspace_bytes(*args[:5], S, i32(cu), max_len=T), dtype=torch.uint8,
                         device=args[0].device)
        sf.gdn_ragged_fwd(*args[:5], S, i32(cu), max_len=T, out=(o, ws))
        torch.cuda.synchronize()
        assert bool((o[torch.tensor(~named, device=o.device)] == 7).all())
        idle = [i for i in range(N + 1) if i == N or at[i + 1] <= at[i]]
        assert torch.equal(S[idle], args[5][idle])
