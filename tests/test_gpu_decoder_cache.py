"""The example's cache is asked for more tokens than it has room for."""
import pytest
import torch

import example_decoder as ex

pytestmark = pytest.mark.gpu


def test_a_full_cache_says_so_and_stays_as_it_was(dnb):
    block = ex.Block(40, 96, 6, 2, torch.float32, seed=3)
    cache = ex.Cache(block, 3, 4)
    token = torch.tensor([1, 2, 3], device="cuda")
    for _ in range(4):
        cache.next(token)
    k, v, lengths = cache.k.clone(), cache.v.clone(), cache.lengths.clone()
    with pytest.raises(ValueError):
        cache.next(token)
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v) and torch.equal(cache.lengths, lengths)
    cache.close()
