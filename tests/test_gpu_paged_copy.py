"""Copying of pages on the device, bit for bit."""
import numpy as np
import pytest
import torch

from paged_util import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page_bytes", [16, 48, 4096, 16384, 16400, 32768, 65520])
@pytest.mark.parametrize("planes,gap", [(1, 0), (3, 0), (4, 4096)])
def test_pages_are_copied(dnb, page_bytes, planes, gap):
    pages = 40
    stride = pages * page_bytes + gap
    pool = torch.randint(0, 256, (planes * stride,), dtype=torch.uint8, generator=torch.Generator().manual_seed(page_bytes)).cuda()
    want = pool.clone()
    order = np.random.default_rng(planes).permutation(pages)
    pairs = order[:22].reshape(11, 2).astype(np.int32)
    for i in range(planes):
        plane = want[i * stride:i * stride + pages * page_bytes].view(pages, page_bytes)
        plane[torch.tensor(pairs[:, 1].astype(np.int64)).cuda()] = plane[torch.tensor(pairs[:, 0].astype(np.int64)).cuda()].clone()
    # pairs that are not of the pool, or twice one page, do nothing
    more = np.concatenate([pairs, [[-1, -1], [order[30], pages], [2 ** 31 - 1, order[31]], [order[32], order[32]], [-5, order[33]]]]).astype(np.int32)
    dnb.dnb_op_paged_copy(pool, pages, page_bytes, planes, stride, ints(more), len(more))
    assert torch.equal(pool, want)


def test_past_32_bits(dnb):
    page_bytes, pages = 1 << 20, 5000
    pool = torch.zeros(pages, page_bytes, dtype=torch.uint8, device="cuda")
    pool[7] = 3
    pool[4998] = 9
    dnb.dnb_op_paged_copy(pool, pages, page_bytes, 1, pages * page_bytes, ints([[7, 4999], [4998, 2]]), 2)
    assert (pool[4999] == 3).all() and (pool[2] == 9).all() and int(pool.sum(dtype=torch.int64)) == 24 * page_bytes


def test_in_a_graph_with_lists_that_change(dnb):
    pool = torch.arange(64, device="cuda", dtype=torch.float32)[:, None].repeat(1, 64).contiguous()
    pairs = ints([[-1, -1]] * 4)
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            dnb.dnb_op_paged_copy(pool, 64, 256, 1, 64 * 256, pairs, 4)
    want = pool.clone()
    for step in ([[1, 2]], [[2, 9], [3, 10]], [], [[9, 0], [60, 63], [4, 5], [7, 8]]):
        pairs.fill_(-1)
        if step:
            pairs[:len(step)] = ints(step)
            for a, b in step:
                want[b] = want[a]
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(pool, want)
