"""Queries with a channel far larger than the others, as attention's inputs have them, against keys that are zero or weak just there: what the small
channels add up to decides, and none of their bits may go.  The bound is that of sums in fp32 (kv_util.compare)."""
import numpy as np
import pytest

from kv_util import Batch

pytestmark = pytest.mark.gpu


def outliers(b, factor, weak, channel):
    """One channel of every query `factor` times as large; keys four times as large as Batch's but at that channel, where they are zero, or,
    with `weak`, in its whole block 2^-20 of that."""
    b.q[:, :, channel] = np.where(b.q[:, :, channel] < 0, -factor, factor)
    page, dim = b.page, b.dim
    half, tail = page * dim // 2, page * dim // 32
    codes = b.data[:, :, :half].reshape(*b.data.shape[:2], page, dim // 2)
    scales = b.data[:, :, 2 * half:2 * half + tail].reshape(*b.data.shape[:2], page, dim // 32)
    scales[scales != 255] += 2
    if weak:
        block = scales[..., channel // 32]
        block[block != 255] -= 20
    else:
        codes[..., channel // 2] &= 0x0f if channel % 2 else 0xf0
    return b


@pytest.mark.parametrize("weak", (False, True))
@pytest.mark.parametrize("factor", (2.0 ** 8, 2.0 ** 12, 2.0 ** 14, 2.0 ** 17))
@pytest.mark.parametrize("dim", (64, 128))
def test_one_token_each(gpu_device, dim, factor, weak):
    for dtype in ("bf16", "f32"):
        b = Batch(dim + int(factor), [200, 77, 33, 130], [1, 1, 1, 1], 2, 4, dim, 32, dtype)
        outliers(b, factor, weak, 37).check(scale=0.5)


@pytest.mark.parametrize("weak", (False, True))
@pytest.mark.parametrize("factor", (2.0 ** 8, 2.0 ** 12, 2.0 ** 14, 2.0 ** 17))
@pytest.mark.parametrize("dim", (64, 128))
def test_a_prompt(gpu_device, dim, factor, weak):
    """More than 512 rows: the kernel for many queries."""
    b = Batch(dim + int(factor) + 1, [150], [17], 1, 32, dim, 16)
    outliers(b, factor, weak, 20).check(scale=0.5)
