"""The paged cache's operators together, as a decoder uses them: pages' books, writing of new tokens, attention over the pages, forks and
their copies, pages given back and moved together.  Against the same block in 64 bits on whole texts (see test_gpu_decoder_example.py for the
bound of fp32), and operator by operator in bf16."""
import numpy as np
import pytest
import torch

import example_decoder as ex
from paged_util import ints
from seq_util import assert_within, attn_forward
from test_gpu_decoder_example import plain

pytestmark = pytest.mark.gpu


def last_logits(block, texts):
    """Of whole texts, in 64 bits."""
    tokens = torch.tensor([t for text in texts for t in text])
    lengths = [len(t) for t in texts]
    logits = plain(block, tokens, torch.zeros_like(tokens), torch.ones(len(tokens)), lengths)[2]
    return logits[torch.tensor(np.cumsum(lengths) - 1)]


class Texts:
    """A PagedCache beside the texts that it should hold."""

    def __init__(self, block, cache, seed):
        self.block, self.cache, self.rng = block, cache, np.random.default_rng(seed)
        self.texts = [[] for _ in range(cache.requests)]

    def next(self, counts):
        new = [self.rng.integers(0, self.block.symbols, n).tolist() for n in counts]
        got = self.cache.next(new).double().cpu()
        for text, t in zip(self.texts, new):
            text.extend(t)
        want = last_logits(self.block, [text for text, n in zip(self.texts, counts) if n])
        assert got.shape == want.shape
        assert float((got - want).abs().max()) <= 1e-4 * float(want.abs().max())

    def fork(self, a, b):
        self.cache.fork(a, b)
        self.texts[b] = list(self.texts[a])

    def cut(self, a, length=0):
        self.cache.cut(a, length)
        del self.texts[a][length:]


@pytest.mark.parametrize("page", [1, 8, 16])
def test_requests_come_fork_go_and_are_moved(dnb, page):
    block = ex.Block(40, 96, 6, 2, torch.float32, seed=5)
    cache = ex.PagedCache(block, 5, 200, 512 // page, page)
    t = Texts(block, cache, 6)
    t.next([37, 0, 90, 3, 0])        # prompts
    t.next([1, 0, 1, 1, 0])
    t.fork(2, 1)
    t.next([1, 1, 1, 0, 0])          # both go on, each its own way
    t.next([1, 5, 1, 20, 0])
    t.fork(1, 4)
    t.cut(0)                         # its pages are free
    t.cut(2, 50)
    cache.compact()
    t.next([0, 1, 1, 1, 1])
    t.next([66, 1, 30, 1, 2])        # a new prompt beside the others
    t.cut(1)
    t.cut(3, 1)
    cache.compact()
    t.next([1, 10, 1, 1, 1])
    for s in range(5):
        t.cut(s)
    assert cache.free() == cache.layout.pages
    cache.close()


def test_no_room_leaves_all_as_it_was(dnb):
    block = ex.Block(40, 96, 6, 2, torch.float32, seed=7)
    cache = ex.PagedCache(block, 3, 64, 8, 8)
    t = Texts(block, cache, 8)
    t.next([30, 9, 0])
    t.fork(0, 2)
    free = cache.free()
    assert free == 2
    with pytest.raises(dnb.DnbError):   # the fork's own last page and two for the second request
        cache.next([[], [1] * 9, [2] * 3])
    t.next([1, 1, 0])
    t.next([1, 0, 1])
    cache.close()


def test_a_captured_step_follows_the_requests(dnb):
    """One graph writes a token of each request and attends to the pages; the host changes lengths, table and rows between its replays,
    among them a request that has none, and forks and copies pages beside it."""
    requests, heads, kv, dim, page, pages, columns = 4, 8, 2, 64, 16, 64, 12
    gen = torch.Generator().manual_seed(9)
    layout = dnb.dnb_paged_layout(pages, page, kv, dim, requests, columns)
    pool = torch.full((2, pages, page, kv, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    w_q, w_k = (torch.rand(dim, generator=gen).cuda() + 0.5 for _ in range(2))
    turns = (10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)).cuda()
    books = dnb.dnb_pages_create(pages, page, requests, columns)
    width = (heads + 2 * kv) * dim

    def make(rows):
        """Tensors and a plan of steps with that many rows, and the step."""
        x = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
        q, k, v = x.split([heads * dim, kv * dim, kv * dim], 1)
        qk = dnb.dnb_qk_layout(rows, heads, kv, dim, dim, q_stride=width, k_stride=width, v_stride=width)
        plan = dnb.dnb_paged_attn_create(layout, heads, rows)
        ws = torch.empty(dnb.dnb_paged_attn_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
        qo, kl, table = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (requests + 1, requests, requests * columns))
        q_out, out = (torch.zeros(rows, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lse = torch.zeros(heads, rows, device="cuda")

        def step():
            dnb.dnb_op_paged_append(qk, layout, q, k, v, w_q, w_k, None, turns, qo, kl, table, q_out, *pool)
            dnb.dnb_paged_attn_forward(plan, q_out, *pool, qo, kl, table, out, lse, ws)
        return x, qo, kl, table, q_out, out, lse, step, plan
    past = [(torch.zeros(0, kv, dim, dtype=torch.bfloat16), torch.zeros(0, kv, dim, dtype=torch.bfloat16)) for _ in range(requests)]

    def run(made, counts, call):
        x, qo, kl, table, q_out, out, lse = made[:7]
        for s, n in enumerate(counts):
            dnb.dnb_pages_extend(books, s, n)
        pairs = dnb.dnb_pages_copies(books)
        plane = pool[0].nbytes
        if len(pairs):
            dnb.dnb_op_paged_copy(pool, pages, plane // pages, 2, plane, torch.from_numpy(pairs).cuda(), len(pairs))
        t, lengths = dnb.dnb_pages_table(books, requests, columns)
        rows = sum(counts)
        x.copy_(torch.randn(x.shape, generator=gen).to(torch.bfloat16))
        qo.copy_(ints(np.cumsum([0] + counts)))
        kl.copy_(ints(lengths))
        table.copy_(ints(t.ravel()))
        out.fill_(9)
        call()
        torch.cuda.synchronize()
        # keys as the same pass without pages makes them
        k_out, other = torch.empty(rows, kv, dim, dtype=torch.bfloat16, device="cuda"), torch.empty_like(q_out[:rows])
        pos = ints(np.concatenate([np.arange(n - c, n) for n, c in zip(lengths, counts)]))
        q, k, v = x[:rows].split([heads * dim, kv * dim, kv * dim], 1)
        dnb.dnb_op_qk_rope_forward(dnb.dnb_qk_layout(rows, heads, kv, dim, dim, q_stride=width, k_stride=width), q, k, w_q, w_k, pos, turns, other, k_out)
        assert torch.equal(other, q_out[:rows])
        at = 0
        for s, c in enumerate(counts):
            past[s] = tuple(torch.cat([a, b[at:at + c].cpu().reshape(c, kv, dim)]) for a, b in zip(past[s], (k_out, v)))
            at += c
        assert [len(a) for a, _ in past] == list(lengths)
        offs = np.cumsum([0] + [len(a) for a, _ in past])
        want, lwant, tol, ltol = attn_forward(q_out[:rows].cpu(), torch.cat([a for a, _ in past]), torch.cat([b for _, b in past]),
                                              np.cumsum([0] + counts), offs, None, True)
        assert_within(out[:rows], want, tol, "out")
        assert_within(lse[:, :rows], lwant, ltol, "lse")
        assert (out[rows:] == 9).all()

    chunk, token = make(120), make(requests)
    run(chunk, [70, 0, 33, 16], chunk[7])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    run(token, [1, 1, 1, 1], token[7])
    side.wait_stream(torch.cuda.current_stream())
    # (a captured call does nothing yet)
    with torch.cuda.graph(graph, stream=side):
        token[7]()
    for _ in range(4):
        run(token, [1, 1, 1, 1], graph.replay)
    dnb.dnb_pages_truncate(books, 1, 0)
    past[1] = tuple(t[:0] for t in past[1])
    run(token, [1, 0, 1, 0], graph.replay)
    dnb.dnb_pages_fork(books, 0, 1)
    past[1] = past[0]
    for _ in range(3):
        run(token, [1, 1, 0, 1], graph.replay)
    run(chunk, [1, 40, 20, 0], chunk[7])
    dnb.dnb_pages_truncate(books, 0, 20)
    past[0] = tuple(t[:20] for t in past[0])
    dnb.dnb_pages_compact(books)
    for _ in range(3):
        run(token, [1, 1, 1, 1], graph.replay)
    for made in (chunk, token):
        dnb.dnb_paged_attn_destroy(made[8])
    dnb.dnb_pages_destroy(books)
