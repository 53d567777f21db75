"""Attention over expanded keys and values at the edges of its calls."""
import pytest
import torch

import paper_2405_12591_amd as dq
from paged_util import DEV, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [128, 64])
def test_rows_without_a_token_in_the_batch_are_zeros(d):
    q, kv, kr = (torch.ones(shape, dtype=torch.bfloat16, device=DEV) for shape in ((5, 3, d + d // 2), (0, 3, 2 * d), (0, d // 2)))
    for causal in (True, False):
        out = torch.full((5, 3, d), 7.0, dtype=torch.bfloat16, device=DEV)
        dq.expanded_attention(q, kv[..., :d], kr, kv[..., d:], ints([1, 3, 4]), ints([0, 0, 0]), 2, 0, dq.expanded_workspace(2, 5, 3, d, 2, 0), out=out, causal=causal)
        assert not out[1:4].any() and bool((out[[0, 4]] == 7).all())
