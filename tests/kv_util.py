"""Caches, tables and comparisons shared by the tests of the paged 4-bit cache."""
import numpy as np
import torch

import paper_2503_06823_amd as P
from oracle import kv_cache as ref

EPS32 = 2.0 ** -24


def bf16(x):
    """fp64 images of bf16 numbers near x"""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


def as_device(x, dtype):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    return t.cuda()


def page_bytes(page, dim):
    return page * dim * 17 // 16


class Batch:
    """Requests with their tokens in a cache whose other bytes are NaN blocks and noise."""

    def __init__(self, seed, lengths, news, kv_heads, group, dim, page, dtype="bf16", spare=2, strong=1.0):
        g = np.random.default_rng(seed)
        self.lengths, self.news, self.page, self.dim, self.dtype = lengths, news, page, dim, dtype
        self.kv_heads, self.q_heads = kv_heads, kv_heads * group
        need = [-(-max(n, 0) // page) for n in lengths]
        pages = sum(need) + spare
        self.data = g.integers(0, 256, (pages, kv_heads, page_bytes(page, dim)), dtype=np.uint8)
        self.data[:, :, page * dim:] = 255  # never written: NaN
        self.cache = ref.Cache(self.data, page, dim)
        width = max(max(need, default=0), 1) + 1
        self.table = np.full((max(len(lengths), 1), width), -1, dtype=np.int32)
        ids, at = g.permutation(pages), 0
        for r, n in enumerate(need):
            self.table[r, :n] = ids[at:at + n]
            at += n
        for r, n in enumerate(lengths):
            for j in range(max(n, 0)):
                slot = int(self.table[r, j // page]) * page + j % page
                for which in (0, 1):
                    codes = g.integers(0, 16, (kv_heads, dim), dtype=np.uint8)
                    scales = g.integers(124, 127, (kv_heads, dim // 32), dtype=np.uint8)
                    self.cache.write(slot, which, codes, scales)
        self.T = sum(news)
        self.cu = np.concatenate(([0], np.cumsum(news))).astype(np.int32)
        q = g.standard_normal((self.T, self.q_heads, dim)) * strong
        self.q = bf16(q) if dtype == "bf16" else q.astype(np.float32).astype(np.float64)

    def slot(self, r, j):
        return int(self.table[r, j // self.page]) * self.page + j % self.page

    def kv(self):
        return P.make_kv_desc(self.data.shape[0], self.page, self.kv_heads, self.dim, len(self.lengths), self.table.shape[1])

    def run(self, window=0, sinks=0, scale=None, max_new=None, gap=0, stream=None, ws_fill=None):
        """emoe_kv_attention into a buffer of 7s; returns the whole of it [T + 3, q_heads * D + gap] and the rows' view."""
        row = self.q_heads * self.dim
        q = torch.full((self.T, row + gap), 9.0, device="cuda").to(torch.float32 if self.dtype == "f32" else torch.bfloat16)
        q[:, :row] = as_device(self.q.reshape(self.T, row), self.dtype)
        out = torch.full((self.T + 3, row + gap), 7.0, device="cuda", dtype=q.dtype)
        kv = self.kv()
        at = P.make_attention_desc(self.T, self.q_heads, self.dim, self.dtype, max(self.news) if max_new is None else max_new, window, sinks,
                                   scale, row + gap, row + gap)
        n = P.emoe_kv_attention_workspace_bytes(kv, at)
        assert n <= 64 << 20
        ws = torch.full((n,), 255 if ws_fill is None else ws_fill, dtype=torch.uint8, device="cuda")
        args = (torch.from_numpy(self.data).cuda(), torch.from_numpy(self.table).cuda(),
                torch.tensor(self.lengths, dtype=torch.int32, device="cuda"), torch.from_numpy(self.cu).cuda())
        torch.cuda.synchronize()
        P.emoe_kv_attention(kv, at, q, *args, out, ws, n, stream)
        torch.cuda.synchronize()
        assert (out[self.T:] == 7.0).all() and (out[:, row:] == 7.0).all()
        return out[:self.T, :row].double().cpu().numpy().reshape(self.T, self.q_heads, self.dim)

    def check(self, window=0, sinks=0, scale=None, **kw):
        got = self.run(window, sinks, scale, **kw)
        want, seen = ref.attention(self.cache, self.q, self.table, self.lengths, self.cu, self.dim ** -0.5 if scale is None else scale, window, sinks)
        compare(got, want, seen, self.dim, self.dtype)
        return got


def compare(got, want, seen, dim, dtype):
    """Element-wise, against a bound from the arithmetic: scores are sums of dim products in fp32 (and one more rounding for the
    scale and the difference each), an error d of all scores changes a weighted mean of values by at most 2 d max|v|; weights and sums of
    n terms add n + 8 roundings; bf16 rounds each weight and the result once more to 8 bits."""
    v_max, qk, n = seen
    rel = 2.0 * (dim + 8) * EPS32 * (qk + 1.0) + (n + 8.0) * 2.0 * EPS32
    if dtype == "bf16":
        rel = rel + 2.0 ** -9 + 2.0 ** -9
    bound = (v_max * rel)[:, :, None] + 1e-37
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    off = np.abs(np.where(nan, 0.0, got - np.where(nan, 0.0, want)))
    off = np.where(nan, 0.0, off)
    assert (off <= np.broadcast_to(np.where(np.isnan(bound), np.inf, bound), off.shape)).all(), float((off / bound).max())
