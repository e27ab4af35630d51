"""What packed_paths.py says about the choice of kernels, against the workspaces that the library wants: partial sums are part of them
where a product runs in tiles."""
import itertools

import pytest

import paper_2503_06823_amd as P
from packed_paths import CUT_FROM, SHORT, blocks, experts_take_tiles, takes_tiles

PLAN = 256  # bytes of a product in tiles; rows are counted to the byte
SUMS = PLAN + (64 << 20)  # and of one that is cut along K


def row_bytes(at, rows, K):
    for n in (rows * blocks(K) * 128, rows * -(-blocks(K) // 4) * 4):
        at = -(-(at + n) // 256) * 256
    return at


EXTENTS = [128, 136, 264, 520, 1032, 1416, 2056, 3208, 4096, 14336]


@pytest.mark.parametrize("groups", (1, 2, 3, 8, 24, 64))
def test_products(groups):
    tiled = 0
    for N, K, rows in itertools.product(EXTENTS, EXTENTS, (1, 16, 64, 65, 200, 48 * groups, 48 * groups + 1, 1000, 1025, 3000, 8192, 20000)):
        if (rows + 2) * max(blocks(N), blocks(K)) * 128 <= 1 << 31:
            more = P.emoe_matmul_workspace_bytes(P.make_matmul_desc(rows, N, K, groups)) - row_bytes(0, rows, K)
            assert more == (0 if not takes_tiles(rows, groups, N, K) else SUMS if blocks(K) >= CUT_FROM else PLAN), (rows, groups, N, K)
            tiled += more > 0
    assert tiled > 100


@pytest.mark.parametrize("act", ("swiglu", "relu"))
@pytest.mark.parametrize("S,k", [(1, 1), (2, 1), (3, 2), (6, 2), (24, 6), (64, 8)])
def test_experts(S, k, act):
    seen = set()
    for d, f, T in itertools.product(EXTENTS, EXTENTS, (1, 16, 64, 65, 48 * S, 600, 1000, 1500, 3000, 4100, 8192)):
        if (T * k + 2) * max(blocks(d), blocks(f)) * 128 <= 1 << 31:
            n = P.emoe_workspace_bytes(P.make_desc(T, d, f, S, k, S, "f8", act))[1]
            at = row_bytes(row_bytes(0, T * k, f), T * k, d)
            both = experts_take_tiles(T, d, f, S, k)
            if both[0] and blocks(f) <= SHORT:
                at = -(-(at + T * k * blocks(f) * 16) // 256) * 256
            cut = any(tiled and blocks(K) >= CUT_FROM for tiled, K in zip(both, (d, f)))
            assert n - at == (SUMS if cut else PLAN if any(both) else 0), (T, d, f, S, k)
            seen.add(both)
    assert len(seen) == 4
