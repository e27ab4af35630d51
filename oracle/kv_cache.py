"""Paged 4-bit key/value cache and attention over it, in plain numpy and 64 bits: the definitions that include/emoe.h states, one
request, one page, one block at a time.  Shares no code with the library.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32
CODE_VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def scale_exponent(amax: float) -> int:
    """The smallest k of -126 .. 125 with amax <= 7 * 2^k, 125 if there is none: 6 * 2^125 is below 2^128, 4 * 2^126 is not."""
    if amax == 0.0:
        return -126
    k = math.frexp(amax)[1] - 5  # amax >= 2^(k+4): too small for sure
    while amax > math.ldexp(7.0, k):
        k += 1
    return min(max(k, -126), 125)


def code_of(x: float) -> int:
    """The code nearest to x, ties to the even code, beyond 6 the 6; the sign in bit 3."""
    a = abs(x)
    best = min(range(8), key=lambda c: (abs(CODE_VALUES[c] - a), c % 2))
    return best + (8 if math.copysign(1.0, x) < 0 else 0)


def quantise(rows: np.ndarray):
    """rows [..., D] (fp64 images of the storage type) -> codes uint8 [..., D], scale bytes uint8 [..., D / 32]."""
    flat = np.asarray(rows, dtype=np.float64).reshape(-1, BLOCK)
    codes = np.zeros(flat.shape, dtype=np.uint8)
    scales = np.zeros(flat.shape[0], dtype=np.uint8)
    for i, b in enumerate(flat):
        if not np.isfinite(b).all():
            scales[i] = 255
            continue
        k = scale_exponent(float(np.abs(b).max()))
        scales[i] = k + 127
        codes[i] = [code_of(math.ldexp(float(x), -k)) for x in b]
    return codes.reshape(rows.shape), scales.reshape(*rows.shape[:-1], rows.shape[-1] // BLOCK)


def numbers(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    v = CODE_VALUES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(s, BLOCK, axis=-1)


class Cache:
    """The bytes of a cache [pages][kv_heads][page bytes], written and read a token at a time."""

    def __init__(self, data: np.ndarray, page: int, dim: int):
        self.data, self.page, self.dim = data, page, dim
        self.codes, self.scales = page * dim // 2, page * dim // BLOCK

    def _spans(self, slot: int, which: int):
        p, at = divmod(slot, self.page)
        c = which * self.codes + at * self.dim // 2
        s = 2 * self.codes + which * self.scales + at * self.dim // BLOCK
        return p, slice(c, c + self.dim // 2), slice(s, s + self.dim // BLOCK)

    def write(self, slot: int, which: int, codes, scales):
        """codes [kv_heads, D], scales [kv_heads, D / 32]; which: 0 keys, 1 values"""
        p, c, s = self._spans(slot, which)
        self.data[p, :, c] = codes[:, 0::2] | (codes[:, 1::2] << 4)
        self.data[p, :, s] = scales

    def read(self, slot: int, which: int) -> np.ndarray:
        p, c, s = self._spans(slot, which)
        b = self.data[p, :, c]
        return numbers(np.stack((b & 15, b >> 4), -1).reshape(b.shape[0], self.dim), self.data[p, :, s])


def plan(page, width, T, length, new_len, table, ring, counters):
    """The tables of a step; returns a dict of what emoe_kv_plan writes (the table as a copy)."""
    table, R, pages = table.copy(), len(length), len(ring)
    head, tail = int(counters[0]), int(counters[1])
    cu, slot, position, seq, taken, wanted, refused = [0], [-1] * T, [-1] * T, [], 0, 0, 0
    for r in range(R):
        l, n = max(int(length[r]), 0), max(int(new_len[r]), 0)
        have, want = -(-l // page), -(-(l + n) // page)
        fits = want <= width and cu[-1] + n <= T
        need = want - have if fits else 0
        wanted += need
        ok = fits and (need == 0 or wanted <= tail - head)
        if ok:
            for i in range(need):
                table[r, have + i] = ring[(head + taken) % pages]
                taken += 1
        else:
            refused += 1
        for i in range(n):
            if cu[-1] + i < T:
                position[cu[-1] + i] = l + i
                if ok:
                    p = int(table[r, (l + i) // page])
                    slot[cu[-1] + i] = p * page + (l + i) % page if 0 <= p < pages else -1
        seq.append(l + n if ok else 0)
        cu.append(cu[-1] + n)
    return dict(table=table, cu=cu, slot=slot, position=position, seq_len=seq, counters=[head + taken, tail], refused=refused)


def release(page, length_before, length, ended, window, sinks, table, ring, counters):
    """The ring (a copy) and the counters after emoe_kv_release."""
    ring, tail = ring.copy(), int(counters[1])
    if length_before is not None:  # a refused row holds what it held
        length = np.maximum(length, length_before)

    def dead(b, n):  # no query at position n or later sees a token of page b
        return all(j >= sinks and j <= n - window for j in range(b * page, (b + 1) * page)) and b * page >= sinks if window else False

    for r in range(len(length)):
        for b in range(-(-max(int(length[r]), 0) // page)):
            gone = window and dead(b, int(length_before[r]))
            if not gone and (ended is not None and ended[r] or dead(b, int(length[r]))):
                ring[tail % len(ring)] = table[r, b]
                tail += 1
    return ring, [int(counters[0]), tail]


def advance(length, seq_len, ended):
    """What the requests hold after a step."""
    return [0 if ended is not None and ended[r] else max(int(length[r]), int(seq_len[r])) for r in range(len(length))]


def attention(cache: Cache, q, table, seq_len, cu, scale, window=0, sinks=0):
    """q [T, q_heads, D] fp64.  Returns (out, bound): bound[t, h] = max |v| seen and the largest sum |q_i k_i| * scale seen, for error
    bounds.  Tokens without a page (-1) are not seen."""
    T, q_heads, D = q.shape
    kv_heads = cache.data.shape[1]
    G = q_heads // kv_heads
    out = np.zeros(q.shape)
    v_max, qk, count = np.zeros((T, q_heads)), np.zeros((T, q_heads)), np.zeros((T, q_heads))
    for r in range(len(seq_len)):
        n, L = int(cu[r + 1] - cu[r]), int(seq_len[r])
        if n == 0 or L <= 0:
            continue
        pages = [int(table[r, j // cache.page]) for j in range(L)]
        there = np.array([0 <= p < cache.data.shape[0] for p in pages])
        slots = [p * cache.page + j % cache.page if ok else 0 for j, (p, ok) in enumerate(zip(pages, there))]
        k = np.stack([cache.read(s, 0) for s in slots])  # [L, kv_heads, D]
        v = np.stack([cache.read(s, 1) for s in slots])
        for i in range(n):
            p = L - n + i
            j = np.arange(L)
            sees = there & (j <= p)
            if window:
                sees &= (j > p - window) | (j < sinks)
            at = np.nonzero(sees)[0]
            if not len(at):
                continue
            t = int(cu[r]) + i
            for h in range(q_heads):
                kk, vv = k[at, h // G], v[at, h // G]
                z = scale * (kk @ q[t, h])
                w = np.exp(z - z.max())
                out[t, h] = (w[:, None] * vv).sum(0) / w.sum()
                v_max[t, h] = np.nanmax(np.abs(vv)) if not np.isnan(vv).all() else 0.0
                qk[t, h] = abs(scale) * (np.abs(kk) @ np.abs(q[t, h])).max()
                count[t, h] = len(at)
    return out, (v_max, qk, count)
