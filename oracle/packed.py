"""Matrices in 8 bits and products with them, in plain numpy and 64 bits: the definitions that include/emoe.h states.  Shares no
code with the library.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128
# the 127 non-negative numbers of a code, by code
CODE_VALUES = np.array([(c % 8) * 2.0 ** -9 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127)])
_MIDDLES = (CODE_VALUES[1:] + CODE_VALUES[:-1]) / 2


def scale_exponent(top: float) -> int:
    """The smallest e of -126 .. 119 with top <= 448 * 2^e, 119 if there is none."""
    if top == 0.0:
        return -126
    e = math.frexp(top)[1] - 10  # top >= 2^(e+9): too small for sure
    while top > math.ldexp(448.0, e):
        e += 1
    return min(max(e, -126), 119)


def scale_exponents(top: np.ndarray) -> np.ndarray:
    flat = np.array([scale_exponent(float(t)) for t in np.ravel(top)], dtype=np.int64)
    return flat.reshape(np.shape(top))


def codes_of(x: np.ndarray) -> np.ndarray:
    """The codes nearest to x, ties to the even code, beyond 448 that of 448; the sign in bit 7."""
    a = np.abs(x)
    c = np.searchsorted(_MIDDLES, a, side="left")
    on = (c < len(_MIDDLES)) & (a == _MIDDLES[np.minimum(c, len(_MIDDLES) - 1)])
    c = np.where(on & (c % 2 == 1), c + 1, c)  # halfway between codes c and c + 1
    return (c + 128 * np.signbit(x)).astype(np.uint8)


def values_of(codes: np.ndarray) -> np.ndarray:
    v = CODE_VALUES[np.minimum(codes & 127, 126)]
    return np.where(codes >= 128, -v, v)


def quantise_rows(x: np.ndarray, exponents=None) -> np.ndarray:
    """x [rows, K] -> the numbers that its elements become, each 128 of a row under a power of two."""
    rows, K = x.shape
    out = np.empty_like(x)
    for j in range(0, K, BLOCK):
        b = x[:, j:j + BLOCK]
        fine = np.isfinite(b).all(1)
        e = scale_exponents(np.abs(np.where(fine[:, None], b, 0.0)).max(1)) if exponents is None else exponents[:, j // BLOCK]
        s = np.ldexp(1.0, e)[:, None]
        out[:, j:j + BLOCK] = np.where(fine[:, None], values_of(codes_of(np.where(fine[:, None], b, 0.0) / s)) * s, np.nan)
    return out


def row_exponents(x: np.ndarray) -> np.ndarray:
    return np.stack([scale_exponents(np.abs(x[:, j:j + BLOCK]).max(1)) for j in range(0, x.shape[1], BLOCK)], 1)


def matrix_bytes(N: int, K: int) -> int:
    nb, kb = -(-N // BLOCK), -(-K // BLOCK)
    return nb * kb * BLOCK * BLOCK + -(-nb * (-(-kb // 4) * 4) // 256) * 256


def pack(w: np.ndarray) -> np.ndarray:
    """w [N, K] (fp64 images of the storage type) -> the bytes of the packed matrix; bytes that no extent covers are zero."""
    N, K = w.shape
    nb, kb = -(-N // BLOCK), -(-K // BLOCK)
    out = np.zeros(matrix_bytes(N, K), dtype=np.uint8)
    scales = out[nb * kb * BLOCK * BLOCK:]
    for i in range(nb):
        for j in range(kb):
            b = np.zeros((BLOCK, BLOCK))
            part = w[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK]
            b[:part.shape[0], :part.shape[1]] = part
            at = i * (-(-kb // 4) * 4) + j
            if not np.isfinite(b).all():
                scales[at] = 255
                continue
            e = scale_exponent(float(np.abs(b).max()))
            scales[at] = e + 127
            codes = codes_of(b / math.ldexp(1.0, e)).reshape(8, 16, 2, 4, 16).transpose(0, 2, 3, 1, 4)
            out[(i * kb + j) * BLOCK * BLOCK:(i * kb + j + 1) * BLOCK * BLOCK] = codes.reshape(-1)
    return out


def unpack(data: np.ndarray, N: int, K: int) -> np.ndarray:
    """The numbers [N, K] of a packed matrix."""
    nb, kb = -(-N // BLOCK), -(-K // BLOCK)
    blocks = data[:nb * kb * BLOCK * BLOCK].reshape(nb, kb, 8, 2, 4, 16, 16).transpose(0, 1, 2, 5, 3, 4, 6).reshape(nb, kb, BLOCK, BLOCK)
    scales = data[nb * kb * BLOCK * BLOCK:][:nb * (-(-kb // 4) * 4)].reshape(nb, -1)[:, :kb].astype(np.int64)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, np.where(scales == 255, 0, scales - 127)))
    return (values_of(blocks) * s[:, :, None, None]).transpose(0, 2, 1, 3).reshape(nb * BLOCK, kb * BLOCK)[:N, :K]


def _per_element(exponents: np.ndarray, K: int) -> np.ndarray:
    return np.repeat(np.ldexp(1.0, exponents - 6), BLOCK, 1)[:, :K]


def rows_least(x: np.ndarray) -> np.ndarray:
    """The smallest number that is a normal code in each element's block of the rows."""
    return _per_element(row_exponents(np.where(np.isfinite(x), x, 0.0)), x.shape[1])


def matrix_least(data: np.ndarray, N: int, K: int) -> np.ndarray:
    """The same of a packed matrix."""
    nb, kb = -(-N // BLOCK), -(-K // BLOCK)
    e = data[nb * kb * BLOCK * BLOCK:][:nb * (-(-kb // 4) * 4)].reshape(nb, -1)[:, :kb].astype(np.int64) - 127
    return _per_element(e.repeat(BLOCK, 0)[:N], K)


def product_error(x: np.ndarray, x_least: np.ndarray, w: np.ndarray, w_least: np.ndarray) -> np.ndarray:
    """How far x w^T may be off in the matrix cores, element by element, before the result is rounded.  Products come together in eights, in units
    of 2^-13 of the largest 2^(a + b) among them, a and b the exponents of the two codes (a denormal code has that of the smallest normal one, a
    zero takes no part): each of the seven others loses less than a unit, and 2^(a + b) is at most the product of the two magnitudes, of
    denormal numbers taken as the smallest normal one.  The K / 8 sums and the few that join pieces round to fp32 (2^-23 at most, whichever
    way) relative to no more than the sum of magnitudes."""
    up = lambda v, least: np.where(v == 0, 0.0, np.maximum(np.abs(v), least))
    return up(x, x_least) @ up(w, w_least).T * (7 * 2.0 ** -13 + (x.shape[1] / 8 + 16) * 2.0 ** -23) + 2.0 ** -126


def activation(g: np.ndarray, u=None) -> np.ndarray:
    with np.errstate(over="ignore"):
        return np.maximum(g, 0.0) if u is None else g / (1.0 + np.exp(-g)) * u


def expert_ffn(x: np.ndarray, m1: np.ndarray, m3, m2: np.ndarray, f: int):
    """One expert over rows x [n, d] of 64-bit images of bf16, its matrices as packed bytes.  -> (y [n, d] before its rounding, how far
    each may be off).  An error of h moves its code by a step where a border between two lies within it: the numbers that h less and
    plus its error become bound the one that it becomes, under either scale."""
    d = x.shape[1]
    q, least = quantise_rows(x), rows_least(x)
    product = lambda m, a, a_least, N, K: (a @ unpack(m, N, K).T, product_error(a, a_least, unpack(m, N, K), matrix_least(m, N, K)))
    g, dg = product(m1, q, least, f, d)
    if m3 is None:
        h, dh = activation(g), dg
    else:
        u, du = product(m3, q, least, f, d)
        h = activation(g, u)
        # silu' is within [-0.1, 1.1]; exponential, quotient and product in fp32, a few units each
        silu = activation(g, np.ones_like(g))
        dh = 1.1 * dg * (np.abs(u) + du) + np.abs(silu) * du + np.abs(h) * 2.0 ** -19 + 2.0 ** -126
    largest = row_exponents(np.abs(h) + dh)
    hq = quantise_rows(h)
    off = np.zeros_like(h)
    for e in (row_exponents(np.maximum(np.abs(h) - dh, 0.0)), row_exponents(h), largest):
        for v in (h - dh, h, h + dh):
            off = np.maximum(off, np.abs(quantise_rows(v, e) - hq))
    w2 = unpack(m2, d, f)
    return hq @ w2.T, off @ np.abs(w2).T + product_error(np.where(hq == 0, off, np.abs(hq) + off), _per_element(largest, f), w2, matrix_least(m2, d, f))
