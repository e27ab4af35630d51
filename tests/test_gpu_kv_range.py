"""Values at the ends of the range of fp32: finite inputs give finite results, and what is not finite reaches nobody who does not see it."""
import numpy as np
import pytest

from kv_util import Batch

pytestmark = pytest.mark.gpu


def kernels():
    """Lengths, query tokens and heads of a batch for the kernel for few queries, and for the one for many."""
    return [([60, 40], [3, 1], 4), ([60, 40], [17, 20], 32)]


@pytest.mark.parametrize("dtype,lengths,news,group", [("bf16", *c) for c in kernels()] + [("f32", *kernels()[0])])
@pytest.mark.parametrize("byte", (253, 254))
@pytest.mark.parametrize("dim", (64, 128))
def test_values_beyond_the_range_reach_those_who_see_them_only(gpu_device, dim, byte, dtype, lengths, news, group):
    """Blocks of values whose scale byte lets codes pass fp32's range, at tokens that are masked for some: ahead of a query, behind a window."""
    b = Batch(21, lengths, news, 1, group, dim, 16, dtype)
    clean = b.run(16, 1)
    s = b.slot(0, lengths[0] - 2)  # the last query and the one before see it
    codes = np.full((1, dim), 7, dtype=np.uint8)
    b.cache.write(s, 1, codes, np.full((1, dim // 32), byte, dtype=np.uint8))
    behind = b.slot(0, 20)  # behind every window, and not a sink
    b.cache.write(behind, 1, codes, np.full((1, dim // 32), byte, dtype=np.uint8))
    got = b.run(16, 1)
    n = news[0]
    assert np.isnan(got[n - 2:n]).all()
    unseen = [t for t in range(sum(news)) if not n - 2 <= t < n]
    assert np.array_equal(got[unseen], clean[unseen])
