"""emoe_matmul with many groups of few rows each, where there are just enough rows a group for tiles of 256 x 256, and one group fewer rows than that."""
import numpy as np
import pytest

from packed_paths import takes_tiles
from packed_util import tokens, weights
from test_gpu_matmul import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes,behind,K", [((60,) * 60, 0, 264), ((49,) * 64, 0, 264), ((100, 0, 1, 96, 50, 63, 31) * 9, 33, 3208), ((48,) * 64, 1, 264)])
def test_tiles(gpu_device, sizes, behind, K):
    g = np.random.default_rng(sum(sizes) + K)
    N, rows = 520, sum(sizes) + behind
    assert takes_tiles(rows, len(sizes), N, K)
    check(tokens(g, rows, K), [weights(g, N, K) for _ in sizes], np.concatenate(([0], np.cumsum(sizes))).tolist())


@pytest.mark.parametrize("sizes", [(48,) * 64, (40,) * 60])
def test_streaming(gpu_device, sizes):
    g = np.random.default_rng(len(sizes))
    assert not takes_tiles(sum(sizes), len(sizes), 1040, 264)
    check(tokens(g, sum(sizes), 264), [weights(g, 1040, 264) for _ in sizes], np.concatenate(([0], np.cumsum(sizes))).tolist())
