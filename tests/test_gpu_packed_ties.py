"""Elements of h beside a tie of two codes, where what the matrix cores lose of a sum would decide which of the two an element becomes: every kernel
that makes h gives them the code of the exact sum.  All numbers here are exact in 64 bits, and all that the second product adds is one code."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from oracle import packed as ref
from packed_paths import CUT_FROM, blocks, converts_its_rows, experts_take_tiles
from packed_util import as_device, packed

pytestmark = pytest.mark.gpu

# 16 * 16 + 4 * 4 and + 4 * 12 are the ties 272 (of 256 and 288) and 304 (of 288 and 320).  The third product, 2^-7, is beneath the unit of its
# eight (2^-13 of 2^8, the largest): on the right side of a tie only if it is not lost.
KINDS = [(16, 4, 0.125), (16, 12, -0.125), (16, 4, -0.125), (16, 12, 0.125)]
TIES = [(16, 4, 0.0), (16, 12, 0.0)]


class Beside:
    """One group of columns of eight a token makes its sums; a row's outputs are the sums times 1, 1/2 (ties as well) and 15/16 (none).  With `one_block`
    those of one block of h, another in every expert; the others are far smaller and no ties."""

    def __init__(self, T, d, f, S, k, act, kinds, one_block=False):
        self.T, self.d, self.f, self.S, self.k, self.act = T, d, f, S, k, act
        g = np.random.default_rng(T + d + f)
        x = np.zeros((T, d))
        at = 8 * (1 + np.arange(T) * 5 % (d // 8 - 1))
        kind = np.array(kinds)[np.arange(T) % len(kinds)]
        for i in range(3):
            x[np.arange(T), at + i] = kind[:, i]
        gate = None
        if act == "swiglu":  # silu(32) is 32 in fp32 and 1e-14 less in 64 bits
            x[:, 0] = 8.0
            gate = np.zeros((f, d))
            gate[:, 0] = 4.0
        self.x, self.experts = x, []
        for e in range(S):
            scale = np.array([1.0, 0.5, 0.9375, 1.0, 0.5, 1.0, 1.0])[np.arange(f) % 7]
            columns = np.arange(d) * 13 % f  # of h, that the outputs are
            if one_block:
                here = np.arange(f) // 128 == (7 * e + 3) % blocks(f)
                scale = np.where(here, scale, 0.9375 * 2.0 ** -8)
                its = np.flatnonzero(here)
                columns = np.where(np.arange(d) % 9 == 8, columns, its[np.arange(d) * 5 % len(its)])
            w = np.zeros((f, d))
            for i, v in enumerate((16.0, 4.0, 2.0 ** -4)):
                w[:, 8 + i::8] = v * scale[:, None]
            second = np.zeros((d, f))
            second[np.arange(d), columns] = 1.0
            self.experts.append((w, None, second, columns) if gate is None else (gate, w / 32, second, columns))
        self.slots = np.stack([g.permutation(S)[:k] for _ in range(T)]).reshape(-1)
        self.perm = np.argsort(self.slots, kind="stable")
        self.offsets = np.concatenate(([0], np.cumsum(np.bincount(self.slots, minlength=S))))

    def wanted(self):
        """The numbers that h's elements become, exactly; grouped rows."""
        q = ref.quantise_rows(self.x)
        assert (q == self.x).all()
        out = np.zeros((self.T * self.k, self.d))
        for e, (w1, w3, _, columns) in enumerate(self.experts):
            rows = slice(self.offsets[e], self.offsets[e + 1])
            its = q[self.perm[rows] // self.k]
            out[rows] = ref.quantise_rows(ref.activation(its @ w1.T, None if w3 is None else its @ w3.T))[:, columns]
        return out

    def run(self, grouped=False):
        desc = P.make_desc(self.T, self.d, self.f, self.S, self.k, self.S, "f8", self.act)
        ws = torch.full((P.emoe_workspace_bytes(desc)[1],), 255, dtype=torch.uint8, device="cuda")
        m = [None if self.experts[0][i] is None else packed([e[i] for e in self.experts]) for i in range(3)]
        perm, offsets = (torch.from_numpy(a).int().cuda() for a in (self.perm, self.offsets))
        x, y = as_device(self.x), torch.full((self.T * self.k, self.d), 5.0, dtype=torch.bfloat16, device="cuda")
        if grouped:
            P.emoe_expert_ffn(desc, x[perm.long() // self.k].contiguous(), offsets, *m, y, ws, ws.numel())
        else:
            P.emoe_expert_ffn_gather(desc, x, perm, offsets, *m, y, ws, ws.numel())
        torch.cuda.synchronize()
        return y.double().cpu().numpy()


def check(a, grouped=False):
    want = a.wanted()
    got = a.run(grouped)
    bad = got != want
    assert not bad.any(), f"{int(bad.sum())} of {bad.size}, first at {tuple(np.argwhere(bad)[0])}: {got[bad][0]} for {want[bad][0]}"


# T, d, f, S, k: streaming with rows that it converts itself, and with converted ones of one to four blocks of 16 a stretch
STREAMED = [(4, 264, 520, 3, 2), (16, 1032, 264, 1, 1), (8, 2056, 136, 2, 1), (12, 2056, 1032, 2, 2), (40, 264, 136, 3, 1), (64, 264, 520, 1, 1), (150, 1032, 392, 2, 1),
            (200, 392, 2312, 2, 2)]
# tiles: whole ones, of several groups, of few rows a group; cut along K.  There an element has to matter to its row, which it does if the other blocks are smaller
TILED = [(5300, 264, 520, 1, 1), (8300, 392, 264, 2, 1), (3200, 520, 392, 8, 4), (26000, 136, 104, 1, 1), (5300, 1160, 640, 3, 1), (4300, 3208, 520, 1, 1),
         (2800, 3208, 392, 3, 2), (8200, 520, 136, 3, 2)]


@pytest.mark.parametrize("kinds", (KINDS, TIES + KINDS[:1]), ids=("beside", "on"))
@pytest.mark.parametrize("act", ("relu", "swiglu"))
@pytest.mark.parametrize("T,d,f,S,k", STREAMED)
def test_streamed(gpu_device, T, d, f, S, k, act, kinds):
    assert not experts_take_tiles(T, d, f, S, k)[0]
    if kinds is not KINDS and act == "swiglu":
        kinds = [(16, 4, 0.125), (16, 4, 0.0)]  # (304 in fp32 is a tie, and less in 64 bits)
    check(Beside(T, d, f, S, k, act, kinds))


@pytest.mark.parametrize("grouped", (False, True))
@pytest.mark.parametrize("act", ("relu", "swiglu"))
@pytest.mark.parametrize("T,d,f,S,k", TILED)
def test_tiled(gpu_device, T, d, f, S, k, act, grouped):
    assert experts_take_tiles(T, d, f, S, k)[0]
    check(Beside(T, d, f, S, k, act, KINDS + (TIES if act == "relu" else TIES[:1]), one_block=blocks(f) > 1), grouped)


def test_many_more_elements_than_a_list_holds(gpu_device):
    """All elements of all rows of a block: one workgroup finds tens of thousands."""
    a = Beside(26000, 136, 104, 1, 1, "relu", KINDS)
    assert experts_take_tiles(a.T, a.d, a.f, a.S, a.k)[0]
    for w, _, second, columns in a.experts:
        w[:, 8:] = np.where(w[:, 8:] != 0, np.tile([16.0, 4.0, 2.0 ** -4, 0, 0, 0, 0, 0], a.d // 8 - 1), 0)
    check(a)


def test_the_sizes_are_of_every_kind():
    assert {converts_its_rows(T * k, d) for T, d, f, S, k in STREAMED} == {True, False}
    assert {blocks(d) >= CUT_FROM for T, d, f, S, k in TILED} == {True, False}


def test_the_same_tokens_have_the_same_codes_however_many_stand_beside_them(gpu_device):
    few, many = (Beside(T, 264, 520, 1, 1, "swiglu", KINDS, one_block=True) for T in (40, 5300))
    assert not experts_take_tiles(40, 264, 520, 1, 1)[0] and experts_take_tiles(5300, 264, 520, 1, 1)[0]
    assert (few.x == many.x[:40]).all() and (few.perm == np.arange(40)).all()
    assert (few.run() == many.run()[:40]).all()
