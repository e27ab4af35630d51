"""Values at the ends of the range of fp32: finite inputs give finite results, and what is not finite reaches nobody who does not see it."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from kv_util import Batch, as_device, bf16, compare, page_bytes
from oracle import kv_cache as ref
from test_gpu_kv_attention import large, plain

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


@pytest.mark.parametrize("exponent", (95, 110, 125))
@pytest.mark.parametrize("dim", (64, 128))
@pytest.mark.parametrize("dtype,group", [("bf16", 32), ("bf16", 1), ("f32", 1)])
def test_large_values_have_a_finite_mean(gpu_device, dim, exponent, dtype, group):
    """Values of up to 6 * 2^125 under scores that rise from token to token, stay, or fall: no sum of them on the way passes fp32's range."""
    for steps in (0, 3, -3):
        b = Batch(10, [330], [17], 1, group, dim, 16, dtype)
        for j in range(330):
            s = b.slot(0, j)
            codes = np.zeros((1, dim), dtype=np.uint8)
            codes[0, 0] = 4  # 2 * 2^k along the first axis
            up = 0 if steps == 0 else j // 110 if steps > 0 else 2 - j // 110
            b.cache.write(s, 0, codes, np.full((1, dim // 32), 127 + up, dtype=np.uint8))
            b.cache.write(s, 1, np.full((1, dim), 7, dtype=np.uint8), np.full((1, dim // 32), 127 + exponent, dtype=np.uint8))
        b.q[:, :, 0] = 3.0
        got = b.check(scale=1.0)
        assert np.isfinite(got).all() and (got >= 5.9 * 2.0 ** exponent).all()


@pytest.mark.parametrize("lengths,news,kv_heads,group,dim,dtype", [
    ([30001], [1], 1, 4, 128, "bf16"), ([30001, 700], [1, 1], 1, 8, 64, "bf16"), ([9001], [2], 1, 3, 64, "f32"), ([9000], [520], 1, 1, 64, "bf16"),
    ([9000], [520], 1, 2, 128, "bf16")])
def test_pieces_of_large_values(gpu_device, lengths, news, kv_heads, group, dim, dtype):
    """Requests that are cut along the keys: the sum of their pieces stays in range too."""
    page = 64
    data, table, q = large(5, lengths, news, kv_heads, group, dim, page, dtype)
    half, tail = page * dim // 2, page * dim // 32
    data[:, :, 2 * half + tail:] = 127 + 125  # of values
    kv = P.make_kv_desc(data.shape[0], page, kv_heads, dim, len(lengths), table.shape[1])
    at = P.make_attention_desc(q.shape[0], q.shape[1], dim, dtype, max(news))
    n = P.emoe_kv_attention_workspace_bytes(kv, at)
    ws, out = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    cu = torch.tensor(np.concatenate(([0], np.cumsum(news))), dtype=torch.int32, device="cuda")
    P.emoe_kv_attention(kv, at, q, data, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), cu, out, ws, n)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()
    compare(out.double().cpu().numpy(), *plain(data, table, q, lengths, news, kv_heads, group, dim, page, 0, 0), dim, dtype)


@pytest.mark.parametrize("byte", (5, 12, 20))
@pytest.mark.parametrize("dtype,group", [("bf16", 32), ("bf16", 1), ("f32", 1)])
def test_the_smallest_values_are_not_lost(gpu_device, byte, dtype, group):
    """Values of 2^-123 and more: what they are multiplied with leaves them above the last bit of a subnormal number."""
    b = Batch(11, [330], [17], 1, group, 64, 16, dtype)
    for j in range(330):
        b.cache.write(b.slot(0, j), 1, np.full((1, 64), 4 + j % 4, dtype=np.uint8), np.full((1, 2), byte, dtype=np.uint8))
    got = b.check()
    assert (got > 2.0 ** (byte - 127)).all()


@pytest.mark.parametrize("dim", (64, 128))
@pytest.mark.parametrize("group", (32, 1))
def test_weights_that_add_up_without_a_larger_one(gpu_device, dim, group):
    """Many tokens whose scores are 6, after a first tile of zeros: none is far above the first maximum, their sum is.  Then the same the other way round, and
    rows whose first tiles are behind a window."""
    for low in (range(64), range(64, 2000)):
        b = Batch(31, [2000], [17], 1, group, dim, 64)
        for j in range(2000):
            codes = np.zeros((1, dim), dtype=np.uint8)
            codes[0, 0] = 0 if j in low else 7  # 6
            b.cache.write(b.slot(0, j), 0, codes, np.full((1, dim // 32), 127, dtype=np.uint8))
        b.q[:, :, 0] = 1.0
        b.check(scale=1.0)
        b.check(1930, 1, scale=1.0)
