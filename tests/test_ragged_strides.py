"""Ragged delta rule: operands that must lie alike are compared where they are stepped.
With one token (or one head) a slice of a wider projection and a packed tensor are alike."""
import pytest
import torch

import paper_2608_06838_amd as sf

from test_serve_cpu import gdn_args


def wider(t, dim):
    """t as the first part of a tensor three times as wide along dim."""
    return torch.cat([t, t, t], dim).narrow(dim, 0, t.shape[dim])


@pytest.mark.parametrize("name,dim", [("beta", 1), ("g", 1), ("k", 1), ("q", 1)])
def test_one_token_of_a_wider_row(name, dim):
    args = gdn_args(T=1)
    args[name] = wider(args[name], dim)
    with pytest.raises(ValueError, match="must be on one GPU"):  # host memory: everything before was accepted
        sf.gdn_ragged_fwd(**args)
    args = gdn_args(T=2)
    args[name] = wider(args[name], dim)
    with pytest.raises(ValueError, match="strides"):
        sf.gdn_ragged_fwd(**args)


def test_one_head_of_a_wider_row():
    args = gdn_args(T=6, Hk=1, Hv=1)
    args["k"] = args["k"].expand(6, 1, 64).as_strided((6, 1, 64), (64, 8, 1))
    args["beta"] = args["beta"].as_strided((6, 1), (1, 5))
    with pytest.raises(ValueError, match="must be on one GPU"):
        sf.gdn_ragged_fwd(**args)


@pytest.mark.gpu
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_one_token_against_the_plain_run(io):
    from test_gpu_ragged import gdn_inputs, run_gdn
    print(f"[gdn ragged] {io} one token, slices beside packed tensors", flush=True)
    q, k, v, g, beta, state = gdn_inputs(1, 2, 4, 64, 128, 2, io, seed=81)
    for max_len in (1, 300):
        run_gdn([q, wider(k, 1), v, g, wider(beta, 1), state.clone()], [0, 1], [1], max_len=max_len)
        run_gdn([wider(q, 1), k, wider(v, 1), wider(g, 1), beta, state.clone()], [0, 1], [1], max_len=max_len)
