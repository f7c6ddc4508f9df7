"""What the paged cache of the decoder example holds on to does not grow with the prompts that it has seen."""
import pytest
import torch

import example_decoder as ex

pytestmark = pytest.mark.gpu


def test_prompts_of_any_lengths_share_a_workspace(dnb):
    block = ex.Block(40, 96, 6, 2, torch.float32, seed=3)
    cache = ex.PagedCache(block, 2, 200, 40, 16)
    tokens = torch.randint(0, 40, (90,), generator=torch.Generator().manual_seed(4)).tolist()
    first = cache.next([tokens])
    cache.cut(0)
    held = torch.cuda.memory_allocated()
    for n in range(1, 90):
        cache.next([tokens[:n], tokens[:n // 3]])
        cache.cut(0)
        cache.cut(1)
    # (a workspace of this block is 9 MB and more)
    assert torch.cuda.memory_allocated() <= held + (1 << 20)
    assert torch.equal(cache.next([tokens]), first)
    assert cache.next([[], []]).shape == (0, 40)
    cache.close()
