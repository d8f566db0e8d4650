"""Where the example's cache ends: at the table of angles, and at its capacity."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
from attention_half import AttentionHalf, Generation  # noqa: E402


def test_a_cache_ends_where_it_is_full():
    half = AttentionHalf(width=128, heads=2, kv_heads=2, batch=1, tokens=40, block=32, n_select=2, density=0.3, seed=1)
    x = torch.randn(1, 41, 128, device="cuda:0")
    half.forward(x[:, :40].contiguous())
    for capacity in (39, half.table.shape[0] + 1):
        with pytest.raises(ValueError):
            Generation(half, capacity)
    Generation(half, half.table.shape[0])
    cache = Generation(half, 41)
    cache.token(x[:, 40:].contiguous())
    torch.cuda.synchronize()
    kept = cache.k.clone(), cache.lengths.clone(), cache.sums.clone()
    with pytest.raises(ValueError):
        cache.token(x[:, 40:].contiguous())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, (cache.k, cache.lengths, cache.sums)))
