"""A max_new that is less than what some request brings: its first queries are answered, at their own positions, the others are left alone."""
import numpy as np
import pytest

from kv_util import Batch, compare
from oracle import kv_cache as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths,news,kv_heads,group,most,dtype", [
    ([60, 200], [5, 1], 2, 4, 3, "bf16"), ([60, 200], [5, 1], 2, 4, 1, "f32"), ([40, 70, 33], [40, 2, 30], 1, 2, 21, "bf16"),
    ([200, 90], [60, 17], 1, 40, 20, "bf16"), ([90, 64], [90, 1], 1, 33, 33, "bf16")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (13, 2)])
def test_first_queries_at_their_positions(gpu_device, lengths, news, kv_heads, group, most, dtype, window, sinks):
    b = Batch(sum(lengths), lengths, news, kv_heads, group, 64, 16, dtype)
    want, seen = ref.attention(b.cache, b.q, b.table, b.lengths, b.cu, 64 ** -0.5, window, sinks)
    got = b.run(window, sinks, max_new=most)
    done = np.concatenate([np.arange(n) < most for n in news])
    compare(got[done], want[done], tuple(x[done] for x in seen), 64, dtype)
    assert (got[~done] == 7.0).all() and not done.all()
