"""Gradients of the norms of queries and keys: outputs the call would not write are refused."""
import pytest
import torch

import paper_2608_06838_amd as sf


@pytest.mark.parametrize("which", [2, 3])
def test_weight_gradients_without_weights(which):
    t = [torch.zeros(1, 3, h, 64) for h in (4, 2, 4, 2)]
    out = [*t[:2], None, None, None]
    out[which] = torch.zeros(64)
    with pytest.raises(ValueError, match="there are none"):
        sf.qk_norm_bwd(*t, out=tuple(out))
