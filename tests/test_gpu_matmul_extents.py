"""emoe_matmul on both sides of the sizes at which one kernel takes over from another, cut along K in all ways, and at the largest extents."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from oracle import packed as ref
from packed_util import as_device, close, matmul, packed, tokens, weights
from test_gpu_matmul import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("each", (36, 37, 48, 49, 128, 129))
def test_many_tiles(gpu_device, each):
    """64 groups of one tile in N."""
    g = np.random.default_rng(each)
    sizes = np.full(64, each)
    sizes[3], sizes[4], sizes[9], sizes[10] = 0, 2 * each, 1, 2 * each - 1
    check(tokens(g, int(sizes.sum()), 264), [weights(g, 136, 264) for _ in sizes], np.concatenate(([0], np.cumsum(sizes))).tolist())


@pytest.mark.parametrize("rows", (128, 129))
@pytest.mark.parametrize("N", (2048, 136))
def test_few_tiles(gpu_device, rows, N):
    g = np.random.default_rng(rows + N)
    check(tokens(g, rows, 264), [weights(g, N, 264)])


@pytest.mark.parametrize("kb", (1, 2, 3, 4, 5, 7, 8, 9, 10, 13, 16, 17, 31, 33))
def test_blocks_of_columns(gpu_device, kb):
    """A wavefront takes every fourth block, rows' powers come in fours: every remainder, with the last block cut too."""
    g = np.random.default_rng(kb)
    sizes = (150, 0, 257, 3, 130, 300)
    offsets = np.concatenate(([0], np.cumsum(sizes))).tolist()
    K = 128 * kb - 24
    check(tokens(g, sum(sizes), K), [weights(g, 136, K) for _ in sizes], offsets)


@pytest.mark.parametrize("N", (8, 120, 128, 136, 248, 256, 264, 384, 392, 504))
def test_columns_of_out_that_end_inside_a_tile(gpu_device, N):
    g = np.random.default_rng(N)
    for rows in (20, 290):
        check(tokens(g, rows, 264), [weights(g, N, 264)], out_gap=8)


@pytest.mark.parametrize("sizes", [(2100, 5, 0, 700), (1, 1, 2500)])
def test_rows_of_many_tiles(gpu_device, sizes):
    """More than eight tiles of rows, and groups with hardly any beside them."""
    g = np.random.default_rng(sizes[0])
    check(tokens(g, sum(sizes), 520), [weights(g, 264, 520) for _ in sizes], np.concatenate(([0], np.cumsum(sizes))).tolist())


def block_rows(m, data, nb, K):
    """Block row nb of a packed matrix [N, K] as a packed matrix of its own."""
    kb = -(-K // 128)
    kg, codes = -(-kb // 4), -(-m // 128) * kb * 16384
    part = data[nb * kb * 16384:(nb + 1) * kb * 16384].cpu().numpy(), data[codes + nb * 4 * kg:codes + (nb + 1) * 4 * kg].cpu().numpy()
    return np.concatenate((*part, np.zeros(-len(part[1]) % 256, np.uint8)))


def sample(x, data, N, K, out, rows, nb):
    """Outputs of some rows and one block of 128 columns."""
    some = x[rows].double().cpu().numpy()
    q, one = ref.quantise_rows(some), block_rows(N, data, nb, K)
    n = min(128, N - 128 * nb)
    w = ref.unpack(one, n, K)
    close(out[rows][:, 128 * nb:128 * nb + n], q @ w.T, ref.product_error(q, ref.rows_least(some), w, ref.matrix_least(one, n, K)))


@pytest.mark.parametrize("rows", (2, 30, 140))
def test_the_largest_matrix(gpu_device, rows):
    """Bytes up to 2^31."""
    N, K = 40008, 53248
    g = torch.Generator(device="cuda").manual_seed(rows)
    w = torch.empty((N, K), dtype=torch.bfloat16, device="cuda").normal_(0.0, K ** -0.5, generator=g)
    m = P.PackedMatrices.pack(w)
    del w
    x = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out = m.matmul(x, torch.full((rows, N), float("nan"), dtype=torch.bfloat16, device="cuda"), m.workspace(rows))
    assert not torch.isnan(out).any()
    for nb in (0, 156, 311, 312):
        sample(x, m.data[0], N, K, out, [0, rows // 2, rows - 1], nb)


def test_the_most_rows(gpu_device):
    N, K = 256, 256
    rows = (1 << 23) - 2
    g = torch.Generator(device="cuda").manual_seed(1)
    m = P.PackedMatrices.pack(torch.empty((N, K), dtype=torch.bfloat16, device="cuda").normal_(0.0, K ** -0.5, generator=g))
    x = torch.empty((rows, K), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out = m.matmul(x, torch.full((rows, N), float("nan"), dtype=torch.bfloat16, device="cuda"), m.workspace(rows))
    assert not torch.isnan(out).any()
    for nb in (0, 1):
        sample(x, m.data[0], N, K, out, [0, 1, rows // 2, rows // 2 + 255, rows - 2, rows - 1], nb)
    with pytest.raises(P.EmoeError):
        m.workspace(rows + 1)


@pytest.mark.parametrize("each", (47, 48, 49, 64, 65))
def test_more_tiles(gpu_device, each):
    """65 tiles in all, several matrices: rows for streaming at most, and one more a group, groups with more and with less."""
    g = np.random.default_rng(each)
    sizes = np.array([each, each + 30, 0, each - 30, each])
    offsets = np.concatenate(([0], np.cumsum(sizes))).tolist()
    check(tokens(g, int(sizes.sum()), 264), [weights(g, 3208, 264) for _ in sizes], offsets)


@pytest.mark.parametrize("rows", (64, 65, 128, 129))
def test_one_matrix_of_many_tiles(gpu_device, rows):
    g = np.random.default_rng(rows)
    check(tokens(g, rows, 136), [weights(g, 16648, 136)])


@pytest.mark.parametrize("sizes", [(64, 128, 65, 0, 1), (63, 0, 0, 127, 192), (0, 0, 191, 1, 1), (16, 17, 32, 33, 96, 80)])
@pytest.mark.parametrize("behind", (0, 70))
def test_stretches_of_rows(gpu_device, sizes, behind):
    """Rows of a group in stretches of 64: whole ones, one more and one less, groups without any between them; what lies behind the last stays."""
    g = np.random.default_rng(len(sizes) + behind)
    offsets = np.concatenate(([0], np.cumsum(sizes))).tolist()
    check(tokens(g, sum(sizes) + behind, 520), [weights(g, 200, 520) for _ in sizes], offsets)


@pytest.mark.parametrize("rows", (600, 1024, 1100))
def test_many_stretches_of_one_small_matrix(gpu_device, rows):
    g = np.random.default_rng(rows)
    check(tokens(g, rows, 264), [weights(g, 264, 264)])
    check(tokens(g, rows, 264), [weights(g, 264, 264)], [0, rows - 65])


@pytest.mark.parametrize("rows,K", [(700, 128), (1000, 8), (5000, 64)])
def test_one_block_of_columns(gpu_device, rows, K):
    """All rows are streamed, whatever their number."""
    g = np.random.default_rng(rows)
    check(tokens(g, rows, K), [weights(g, 264, K)])
    check(tokens(g, rows, K), [weights(g, 72, K) for _ in range(3)], [0, rows // 2 + 3, rows // 2 + 3, rows - 10])


def test_offsets_out_of_range_stay_in_bounds(gpu_device):
    """Negative, descending and too large ones: nothing outside of out is written."""
    g = np.random.default_rng(1)
    x, data = as_device(tokens(g, 200, 264)), packed([weights(g, 136, 264) for _ in range(4)])
    for at in ([-5, 3, 2, 100, 1 << 30], [0, 1 << 30, -(1 << 30), 50, 60], [200, 200, 300, 100, 7]):
        out = matmul(x, data, 136, at)  # (looks at what lies around)
        assert out.shape == (200, 136)
