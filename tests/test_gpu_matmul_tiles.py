"""emoe_matmul where there are rows enough for the kernel that works in tiles of 256 x 256 (smaller calls are streamed)."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from oracle import packed as ref
from packed_util import as_device, bf16, close, matmul, numbers, packed, tokens, weights
from test_gpu_matmul import check

pytestmark = pytest.mark.gpu

# 33 stretches of 64 rows times 17 of a matrix's: more than are streamed
ROWS, N = 2100, 1040


@pytest.mark.parametrize("rows", (2100, 2304, 2305, 2559))
@pytest.mark.parametrize("K", (136, 256, 264, 1032))
def test_one_matrix(gpu_device, rows, K):
    g = np.random.default_rng(rows + K)
    check(tokens(g, rows, K), [weights(g, N, K)])


@pytest.mark.parametrize("n", (1040, 1144, 1152, 1160, 1272, 1280, 1288))
def test_columns_of_out_that_end_inside_a_tile(gpu_device, n):
    g = np.random.default_rng(n)
    check(tokens(g, ROWS, 264), [weights(g, n, 264)], out_gap=8)


@pytest.mark.parametrize("sizes,behind", [
    ((300, 2, 0, 129, 1700), 70), ((1, 0, 2200), 0), ((0, 0, 2100), 1), ((2100, 0, 1, 15, 16, 17, 255, 256, 257), 0), ((40,) * 60, 0), ((530, 528, 513, 600), 300)])
@pytest.mark.parametrize("K", (264, 384))
def test_groups(gpu_device, sizes, behind, K):
    g = np.random.default_rng(sum(sizes) + K)
    offsets = np.concatenate(([0], np.cumsum(sizes))).tolist()
    check(tokens(g, sum(sizes) + behind, K), [weights(g, N, K) for _ in sizes], offsets)


@pytest.mark.parametrize("kb", (2, 3, 4, 5, 6, 7, 8, 9, 13, 17, 23, 24, 25, 26, 27, 31, 33))
def test_blocks_of_columns(gpu_device, kb):
    """Tiles are cut along K from 24 blocks on, at whole fours, and rows' powers come in fours: every remainder, with the last block
    cut too."""
    g = np.random.default_rng(kb)
    sizes = (150, 0, 257, 3, 130, 1560)
    offsets = np.concatenate(([0], np.cumsum(sizes))).tolist()
    K = 128 * kb - 24
    check(tokens(g, sum(sizes), K), [weights(g, N, K) for _ in sizes], offsets)


def sampled(x, ws, offsets, got, rows):
    """Some rows of a product."""
    for i in range(len(offsets) - 1):
        mine = rows[(rows >= offsets[i]) & (rows < offsets[i + 1])]
        if len(mine):
            q, w = ref.quantise_rows(x[mine]), numbers(ws[i:i + 1], N, x.shape[1])[0]
            close(got[torch.from_numpy(mine).cuda()], q @ w.T,
                  ref.product_error(q, ref.rows_least(x[mine]), w, ref.matrix_least(ws[i].cpu().numpy(), N, x.shape[1])))


@pytest.mark.parametrize("sizes,K", [((14000, 13000), 264), ((30000,), 136), ((9000, 100, 8000), 3208), ((13300,), 4232), ((13200,), 3336)])
def test_whole_rounds_and_what_is_left_of_them(gpu_device, sizes, K):
    """More tiles than CUs: whole ones, and the rest whole or in pieces."""
    g = np.random.default_rng(K)
    offsets = np.concatenate(([0], np.cumsum(sizes))).tolist()
    x, data = tokens(g, sum(sizes), K), packed([weights(g, N, K) for _ in sizes])
    got = matmul(as_device(x), data, N, offsets)
    assert torch.isfinite(got).all()
    edges = np.concatenate([np.array([a, b - 1]) for a, b in zip(offsets[:-1], offsets[1:])])
    sampled(x, data, offsets, got, np.unique(np.concatenate((edges, g.integers(0, sum(sizes), 300)))))


def test_rows_of_wider_tensors(gpu_device):
    g = np.random.default_rng(4)
    check(tokens(g, ROWS, 392), [weights(g, N, 392)], x_gap=136, out_gap=40)


def test_infinities_and_nan_stay_in_their_rows(gpu_device):
    g = np.random.default_rng(5)
    x, w = tokens(g, ROWS, 264), weights(g, N, 264)
    x[1, 3], x[3, 200], x[ROWS - 1, 263] = np.nan, np.inf, -np.inf
    got = check(x, [w])
    assert set(np.flatnonzero(torch.isnan(got).all(1).cpu().numpy())) == {1, 3, ROWS - 1}
    assert int(torch.isnan(got).any(1).sum()) == 3


def test_magnitudes_from_the_smallest_to_the_largest(gpu_device):
    g = np.random.default_rng(6)
    x, w = tokens(g, ROWS, 512), weights(g, N, 512)
    x[0, :128] *= 2.0 ** -120
    x[1, 128:256] *= 2.0 ** 100
    x[2] *= 2.0 ** -125
    x[3, :] = 0.0
    w[:128, :128] *= 2.0 ** -60
    w[128:256, 256:384] *= 2.0 ** 20
    check(bf16(x), [bf16(w)])


@pytest.mark.parametrize("K", (520, 3336))
def test_repeats_streams_and_replays_give_the_same_bits(gpu_device, K):
    g = np.random.default_rng(K)
    data = packed([weights(g, N, K)])
    xs = [as_device(tokens(g, ROWS, K)) for _ in range(2)]
    want = [matmul(x, data, N).clone() for x in xs]
    for x, w in zip(xs, want):
        assert torch.equal(matmul(x, data, N), w) and torch.equal(matmul(x, data, N), w)
    desc = P.make_matmul_desc(ROWS, N, K)
    room = lambda: torch.empty(P.emoe_matmul_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    streams, ws = [torch.cuda.Stream() for _ in range(2)], [room() for _ in range(2)]
    outs = [torch.empty((ROWS, N), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for i in range(2):
            P.emoe_matmul(desc, xs[i], None, data, outs[i], ws[i], ws[i].numel(), streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))
    held, graph = xs[0].clone(), torch.cuda.CUDAGraph()
    streams[0].wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(streams[0]), torch.cuda.graph(graph, stream=streams[0]):
        P.emoe_matmul(desc, held, None, data, outs[0], ws[0], ws[0].numel())
    for i in (0, 1, 1, 0):
        held.copy_(xs[i])
        outs[0].zero_()
        ws[0].fill_(255 if i else 0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[i])


def test_offsets_out_of_range_stay_in_bounds(gpu_device):
    g = np.random.default_rng(1)
    x, data = as_device(tokens(g, ROWS, 264)), packed([weights(g, N, 264) for _ in range(4)])
    for at in ([-5, 3, 2, 1000, 1 << 30], [0, 1 << 30, -(1 << 30), 50, 60], [ROWS, ROWS, ROWS + 9, 100, 7]):
        assert matmul(x, data, N, at).shape == (ROWS, N)  # (looks at what lies around)
