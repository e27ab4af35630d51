"""Values at the ends of the range of fp32: finite inputs give finite results, and what is not finite reaches nobody who does not see it."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from kv_util import Batch, as_device, bf16, page_bytes
from oracle import kv_cache as ref

pytestmark = pytest.mark.gpu

TOP = {"bf16": float(torch.finfo(torch.bfloat16).max), "f32": float(np.finfo(np.float32).max)}


def cache_of(pages, heads, page, dim):
    return torch.zeros((pages, heads, page_bytes(page, dim)), dtype=torch.uint8, device="cuda")


def read(kv, T, dtype, cache, slots, heads, dim):
    outs = [torch.zeros((T, heads, dim), dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda") for _ in range(2)]
    P.emoe_kv_read(kv, T, dtype, cache, slots, *outs)
    torch.cuda.synchronize()
    return [o.double().cpu().numpy() for o in outs]


@pytest.mark.parametrize("out_type", ("bf16", "f32"))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_the_largest_numbers_stay_numbers(gpu_device, dtype, out_type):
    """Rows up to the type's largest number (its lowest fills masked places): stored, and read back finite."""
    x = np.linspace(-1.0, 1.0, 4 * 128).reshape(4, 1, 128) * np.array([1.0, 0.93, 0.87, 0.5])[:, None, None] * TOP[dtype]
    x[0, 0, 5:9] = -TOP[dtype], TOP[dtype], 1.5 * 2.0 ** 127, -(1.75 * 2.0 ** 127)
    x = bf16(x) if dtype == "bf16" else x.astype(np.float32).astype(np.float64)
    assert np.isfinite(x).all() and np.abs(x).max() == TOP[dtype]
    kv = P.make_kv_desc(1, 16, 1, 128, 1, 1)
    cache, slots = cache_of(1, 1, 16, 128), torch.arange(4, dtype=torch.int32, device="cuda")
    k = as_device(x, dtype)
    P.emoe_kv_append(kv, 4, dtype, k, k, slots, cache)
    for got in read(kv, 4, out_type, cache, slots, 1, 128):
        assert np.isfinite(got).all()
        assert np.array_equal(got, ref.numbers(*ref.quantise(x)))
        assert (np.abs(got - x) <= 0.25 * np.abs(x).max()).all()  # the largest goes to 6 of 8 steps


@pytest.mark.parametrize("out_type", ("bf16", "f32"))
def test_every_scale_and_code(gpu_device, out_type):
    """All 256 scale bytes with all 16 codes, as the format defines them: what passes the output type's range is infinite, what is below it is rounded."""
    page, dim = 256, 64
    data = np.zeros((1, 1, page_bytes(page, dim)), dtype=np.uint8)
    c = ref.Cache(data, page, dim)
    codes = (np.arange(dim) % 16).astype(np.uint8)[None]
    for b in range(256):
        for which in (0, 1):
            c.write(b, which, codes, np.full((1, 2), b, dtype=np.uint8))
    kv = P.make_kv_desc(1, page, 1, dim, 1, 1)
    got = read(kv, page, out_type, torch.from_numpy(data).cuda(), torch.arange(page, dtype=torch.int32, device="cuda"), 1, dim)
    for which in (0, 1):
        want = np.stack([c.read(b, which) for b in range(256)])
        with np.errstate(over="ignore"):
            want = (torch.from_numpy(want).float() if out_type == "f32" else torch.from_numpy(want).to(torch.bfloat16)).double().numpy()
        assert np.array_equal(got[which], want, equal_nan=True)


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


@pytest.mark.parametrize("dtype,lengths,news,group", [("bf16", *c) for c in kernels()] + [("f32", *kernels()[0])])
def test_masked_tokens_of_the_largest_numbers(gpu_device, dtype, lengths, news, group):
    """Tokens whose keys and values are the type's largest and lowest numbers, appended, next to seen ones."""
    b = Batch(22, lengths, news, 1, group, 64, 16, dtype)
    clean = b.run(16, 1)
    kv = b.kv()
    cache = torch.from_numpy(b.data).cuda()
    x = np.full((2, 1, 64), TOP[dtype])
    x[1] = -TOP[dtype]
    k = as_device(x, dtype)
    P.emoe_kv_append(kv, 2, dtype, k, k, torch.tensor([b.slot(0, 19), b.slot(1, 2)], dtype=torch.int32, device="cuda"), cache)
    torch.cuda.synchronize()
    b.data[:] = cache.cpu().numpy()
    assert np.array_equal(b.run(16, 1), clean)
