"""emoe_kv_append and emoe_kv_read: every byte of the cache against the oracle."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from kv_util import as_device, bf16, page_bytes
from oracle import kv_cache as ref

pytestmark = pytest.mark.gpu


def rows_of(g, T, heads, dim, dtype):
    """Rows over many magnitudes, with the values at which rounding and scales turn."""
    x = g.standard_normal((T, heads, dim)) * np.exp(g.uniform(-6, 6, (T, heads, dim // 32)).repeat(32, -1))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 6.0])
    x[0, 0, :16] = ties
    x[0, 0, 16:32] = 0.0
    x[0, -1, 32:64] = np.linspace(-7.0, 7.0, 32)
    x[-1, 0, 32:] = 0.0
    x[-1, 0, 33] = -0.0
    return bf16(x) if dtype == "bf16" else x.astype(np.float32).astype(np.float64)


def append(kv, x, y, slots, cache, dtype, gap=0, stream=None):
    T, row = x.shape[0], x.shape[1] * x.shape[2]
    wide = torch.full((T, 2 * row + gap), float("nan"), dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    wide[:, :row], wide[:, row:2 * row] = as_device(x.reshape(T, row), dtype), as_device(y.reshape(T, row), dtype)
    P.emoe_kv_append(kv, T, dtype, wide, wide[:, row:], torch.tensor(slots, dtype=torch.int32, device="cuda"), cache, 2 * row + gap, 2 * row + gap, stream)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("T,heads,dim,page,gap", [(1, 1, 64, 16, 0), (5, 3, 128, 32, 8), (33, 2, 64, 256, 0), (70, 1, 128, 64, 24), (3, 17, 128, 16, 0)])
def test_append_and_read(gpu_device, T, heads, dim, page, gap, dtype):
    g = np.random.default_rng(T * heads + dim)
    pages = -(-T // page) + 2
    k, v = rows_of(g, T, heads, dim, dtype), rows_of(g, T, heads, dim, dtype)
    slots = g.permutation(pages * page)[:T]
    if T > 4:
        slots[3], slots[4] = -1, pages * page  # nobody's, and beyond the cache
    data = g.integers(0, 256, (pages, heads, page_bytes(page, dim)), dtype=np.uint8)
    cache = torch.from_numpy(data).cuda()
    kv = P.make_kv_desc(pages, page, heads, dim, 1, 1)
    append(kv, k, v, slots, cache, dtype, gap)
    want = ref.Cache(data.copy(), page, dim)
    numbers = [np.zeros_like(k), np.zeros_like(v)]
    for t, s in enumerate(slots):
        if 0 <= s < pages * page:
            for which, x in ((0, k), (1, v)):
                codes, scales = ref.quantise(x[t])
                want.write(int(s), which, codes, scales)
                numbers[which][t] = ref.numbers(codes, scales)
    assert np.array_equal(cache.cpu().numpy(), want.data)
    for out_type in ("bf16", "f32"):
        outs = [torch.full((T + 1, heads, dim), 5.0, dtype=torch.float32 if out_type == "f32" else torch.bfloat16, device="cuda") for _ in range(2)]
        P.emoe_kv_read(kv, T, out_type, cache, torch.tensor(slots, dtype=torch.int32, device="cuda"), *outs)
        torch.cuda.synchronize()
        for o, n in zip(outs, numbers):
            assert np.array_equal(o[:T].double().cpu().numpy(), n) and (o[T] == 5.0).all()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_every_magnitude_and_what_is_not_finite(gpu_device, dtype):
    """One value of every exponent and of many mantissas as the largest of a block, beside blocks that hold an infinity or a NaN."""
    bits = np.arange(0, 0x7f80, 3, dtype=np.uint32) << 16
    tops = bits.view(np.float32).astype(np.float64)
    T = -(-len(tops) // 4)
    x = np.zeros((T, 1, 128))
    flat = x.reshape(-1, 32)
    flat[:len(tops), 5] = tops
    flat[:len(tops), 6] = -tops * 0.375
    flat[:len(tops), 31] = tops / 16
    x = bf16(x) if dtype == "bf16" else x.astype(np.float32).astype(np.float64)
    y = np.ones((T, 1, 128))
    y[1, 0, 40], y[2, 0, 3], y[3, 0, 127] = np.inf, -np.inf, np.nan
    page, pages = 256, -(-T // 256)
    kv = P.make_kv_desc(pages, page, 1, 128, 1, 1)
    cache = torch.zeros((pages, 1, page_bytes(page, 128)), dtype=torch.uint8, device="cuda")
    slots = np.arange(T)
    append(kv, x, y, slots, cache, dtype)
    got = ref.Cache(cache.cpu().numpy(), page, 128)
    want = ref.Cache(np.zeros_like(got.data), page, 128)
    for t in range(T):
        for which, a in ((0, x), (1, y)):
            want.write(t, which, *ref.quantise(a[t]))
    assert np.array_equal(got.data, want.data)
    outs = [torch.zeros((T, 1, 128), dtype=torch.float32, device="cuda") for _ in range(2)]
    P.emoe_kv_read(kv, T, "f32", cache, torch.arange(T, dtype=torch.int32, device="cuda"), *outs)
    torch.cuda.synchronize()
    nan = torch.isnan(outs[1][:, 0]).reshape(T, 4, 32)
    assert nan[1, 1].all() and nan[2, 0].all() and nan[3, 3].all() and nan.sum() == 96


def test_slots_past_four_gigabytes(gpu_device):
    """The last page of a cache of 4.5 GiB: byte offsets beyond 32 bits."""
    heads, dim, page = 8, 128, 256
    per_page = heads * page_bytes(page, dim)
    pages = (9 << 29) // per_page
    kv = P.make_kv_desc(pages, page, heads, dim, 1, 1)
    cache = torch.zeros((pages, heads, page_bytes(page, dim)), dtype=torch.uint8, device="cuda")
    assert P.emoe_kv_cache_bytes(kv) == cache.numel() > 1 << 32
    g = np.random.default_rng(3)
    k, v = rows_of(g, 2, heads, dim, "bf16"), rows_of(g, 2, heads, dim, "bf16")
    append(kv, k, v, [pages * page - 1, 7], cache, "bf16")
    outs = [torch.zeros((2, heads, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    P.emoe_kv_read(kv, 2, "bf16", cache, torch.tensor([pages * page - 1, 7], dtype=torch.int32, device="cuda"), *outs)
    torch.cuda.synchronize()
    for o, x in zip(outs, (k, v)):
        assert np.array_equal(o.double().cpu().numpy(), ref.numbers(*ref.quantise(x)))
    assert not cache[1:-1].any()
