"""Paged caches for the tests: pools in any layout, whose unused rows hold NaN, and what they hold as packed rows."""
import numpy as np
import torch

LAYOUTS = ("tokens", "heads", "turns")


class Cache:
    """Keys and values of `lengths` tokens each in pages of a pool.  layout: tokens first, heads first, or pages of keys and of values
    by turns."""

    def __init__(self, lengths, page, kv_heads, dim, dtype, layout="tokens", seed=0, spare=3, columns=0, scale=1.0):
        self.lengths, self.page, self.kv, self.dim, self.dtype = list(lengths), page, kv_heads, dim, dtype
        need = [-(-n // page) for n in lengths]
        self.pages, self.columns = sum(need) + spare, max(columns, max(need), 1)
        shape = (self.pages, kv_heads, page, dim) if layout == "heads" else (self.pages, page, kv_heads, dim)
        if layout == "turns":
            both = torch.full((self.pages, 2) + shape[1:], float("nan"), dtype=dtype)
            self.k_pool, self.v_pool, self.pool = both[:, 0], both[:, 1], both
            self.strides = dict(page_stride=2 * page * kv_heads * dim, row_stride=kv_heads * dim, head_stride=dim)
        else:
            self.pool = None
            self.k_pool, self.v_pool = (torch.full(shape, float("nan"), dtype=dtype) for _ in range(2))
            self.strides = dict(page_stride=page * kv_heads * dim, row_stride=dim, head_stride=page * dim) if layout == "heads" else {}
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        order = rng.permutation(self.pages)
        # past a sequence's pages the table holds what must never be looked at
        self.table = np.full((len(lengths), self.columns), 2 ** 31 - 1, dtype=np.int32)
        self.k = (torch.randn(sum(lengths), kv_heads, dim, generator=gen) * scale).to(dtype)
        self.v = torch.randn(sum(lengths), kv_heads, dim, generator=gen).to(dtype)
        self.layout, at, used = layout, 0, 0
        for s, n in enumerate(lengths):
            self.table[s, :need[s]] = order[used:used + need[s]]
            used += need[s]
            for j in range(n):
                p, r = int(self.table[s, j // page]), j % page
                where = (p, slice(None), r) if layout == "heads" else (p, r)
                self.k_pool[where] = self.k[at + j]
                self.v_pool[where] = self.v[at + j]
            at += n
        self.k_offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)

    def rows(self, s, first, last):
        """Index of tokens first .. last - 1 of a sequence in a pool, for either layout's first dimensions."""
        j = np.arange(first, last)
        return self.table[s, j // self.page].astype(np.int64), j % self.page

    def to_gpu(self):
        if self.pool is not None:
            g = self.pool.cuda()
            return g[:, 0], g[:, 1]
        return self.k_pool.cuda(), self.v_pool.cuda()

    def layout_of(self, dnb, sequences=None):
        code = dnb.DNB_F32 if self.dtype == torch.float32 else dnb.DNB_BF16
        return dnb.dnb_paged_layout(self.pages, self.page, self.kv, self.dim, sequences or len(self.lengths), self.columns, dtype=code,
                                    **self.strides)


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def offsets(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int64)


def gpu_address(t):
    """Of a view that does not start on its storage."""
    return t.data_ptr()
