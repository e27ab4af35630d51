"""Inputs and comparisons shared by the tests of matrices in 8 bits."""
from __future__ import annotations

import numpy as np
import torch

import paper_2503_06823_amd as P
from oracle import packed as ref

HALF_STEP = 2.0 ** -8  # of bf16, relative to the number that is rounded


def bf16(x):
    """fp64 images of the bf16 numbers nearest to x."""
    return torch.from_numpy(np.ascontiguousarray(x)).float().bfloat16().double().numpy()


def as_device(x, dtype="bf16"):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", torch.float32 if dtype == "f32" else torch.bfloat16)


def weights(g, N, K):
    return bf16(g.standard_normal((N, K)) * np.exp(0.3 * g.standard_normal((N, 1))) * K ** -0.5)


def tokens(g, rows, K):
    """Channels of unequal size, one far above the others."""
    channel = np.exp(0.5 * g.standard_normal(K))
    channel[int(g.integers(K))] *= 20
    return bf16(g.standard_normal((rows, K)) * channel)


def packed(matrices):
    """Packed matrices on the device, by the oracle."""
    return torch.from_numpy(np.stack([ref.pack(w) for w in matrices])).cuda()


def numbers(data, N, K):
    """What packed matrices [count, bytes] stand for."""
    return [ref.unpack(m, N, K) for m in data.cpu().numpy()]


def close(got, want, off):
    """Whether results that were rounded to bf16 are those of sums that are `off` at most from `want`."""
    got = got.double().cpu().numpy()
    both_nan = np.isnan(got) & np.isnan(want)
    bound = off + (np.abs(want) + off) * HALF_STEP + 2.0 ** -133
    bad = ~both_nan & ~(np.abs(got - want) <= bound)
    assert not bad.any(), (f"{int(bad.sum())} of {bad.size} off, first at {tuple(np.argwhere(bad)[0])}: "
                           f"{got[bad][0]} for {want[bad][0]} within {bound[bad][0]}")


def matmul(x, matrices, N, offsets=None, x_gap=0, out_gap=0, stream=None, ws=None, groups=None):
    """x [rows, K] bf16 on the device -> (out rows, what lies between and behind them), all of it 5 before the call."""
    rows, K = x.shape
    wide = torch.full((rows, K + x_gap), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :K] = x
    out = torch.full((rows + 1, N + out_gap), 5.0, dtype=torch.bfloat16, device="cuda")
    groups = (1 if offsets is None else len(offsets) - 1) if groups is None else groups
    desc = P.make_matmul_desc(rows, N, K, groups, "bf16", K + x_gap, N + out_gap)
    if ws is None:
        ws = torch.full((P.emoe_matmul_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")
    at = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    P.emoe_matmul(desc, wide, at, matrices, out, ws, ws.numel(), stream)
    torch.cuda.synchronize()
    assert (out[rows] == 5.0).all() and (out[:rows, N:] == 5.0).all()
    return out[:rows, :N]
