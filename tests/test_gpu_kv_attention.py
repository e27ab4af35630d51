"""emoe_kv_attention against the oracle in 64 bits, element by element within bounds from the arithmetic (kv_util.compare)."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from kv_util import Batch, as_device, compare, page_bytes
from oracle import kv_cache as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("kv_heads,group,dim,page", [(1, 1, 64, 16), (2, 4, 128, 64), (3, 3, 64, 32), (1, 16, 128, 16), (2, 17, 64, 128), (1, 40, 128, 256)])
def test_one_token_each(gpu_device, kv_heads, group, dim, page, dtype):
    """A decode step: lengths of one token, around tiles of 16 and 32, of several pieces."""
    lengths = [1, 2, 15, 16, 17, 31, 32, 33, 64, 100, 129, 257]
    b = Batch(kv_heads * 100 + group, lengths, [1] * len(lengths), kv_heads, group, dim, page, dtype)
    b.check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("lengths,news", [
    ([5], [5]), ([1], [1]), ([40], [40]), ([70], [33]), ([130, 64], [67, 2]), ([3, 200, 17, 40], [3, 1, 17, 20]), ([300], [129]),
    ([20, 0, 65, 90], [0, 0, 65, 0]), ([257, 31], [256, 31]),
])
@pytest.mark.parametrize("kv_heads,group,dim,page", [(2, 4, 128, 16), (1, 5, 64, 64)])
def test_several_tokens(gpu_device, lengths, news, kv_heads, group, dim, page, dtype):
    """Prompts and pieces of prompts next to decoded tokens and to requests without any: causal from their own position on."""
    Batch(len(lengths) + sum(news), lengths, news, kv_heads, group, dim, page, dtype).check(gap=8)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 3), (16, 0), (31, 4), (32, 32), (33, 40), (64, 1), (100, 0), (1000, 7)])
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_window_and_sinks(gpu_device, window, sinks, dtype):
    b = Batch(window + sinks, [1, 20, 33, 150, 230, 400], [1, 7, 33, 1, 66, 2], 2, 3, 64, 16, dtype)
    b.check(window, sinks)
    b = Batch(window + sinks + 1, [333, 90], [1, 1], 1, 8, 128, 32, dtype)
    b.check(window, sinks)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_rows_that_see_nothing_are_zero(gpu_device, dtype):
    """Queries before their request's first token (refused rows: length 0), and requests whose pages belong to nobody."""
    b = Batch(1, [0, 4, 40, 35, -5], [3, 9, 1, 50, 2], 2, 4, 64, 16, dtype)
    b.table[2, :] = -1
    got = b.check()
    cu = b.cu
    assert not got[cu[0]:cu[1]].any() and not got[cu[1]:cu[1] + 5].any() and not got[cu[2]:cu[3]].any() and not got[cu[4]:].any()
    assert got[cu[1] + 5:cu[2]].any()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_pages_of_nobody_inside_a_request_are_not_seen(gpu_device, dtype):
    b = Batch(2, [200, 130, 90], [1, 40, 3], 1, 4, 128, 16, dtype)
    b.table[0, 2], b.table[0, 7], b.table[1, 0], b.table[2, 3] = -1, 1 << 30, -7, b.data.shape[0]
    b.check()
    b.check(20, 3)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("news", ([1], [90]))
def test_lengths_beyond_the_table_stay_in_it(gpu_device, news, dtype):
    """A length of more tokens than the table has entries for: the tokens that it has are seen, at their positions."""
    b = Batch(3, [100], news, 1, 4, 64, 16, dtype)
    b.table = np.ascontiguousarray(b.table[:, :4])
    full = b.table.copy()
    got = b.run()
    b.table = np.concatenate((full, np.full((1, 4), -1, np.int32)), 1)
    want, seen = ref.attention(b.cache, b.q, b.table, b.lengths, b.cu, 64 ** -0.5)
    compare(got, want, seen, 64, dtype)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("which", (0, 1))
def test_what_is_not_a_number_reaches_those_who_see_it_only(gpu_device, which, dtype):
    """NaN blocks of keys or values at tokens that some queries see and others do not: behind a window, ahead of a query, in the
    other requests' pages, in other heads."""
    for group, news, window, sinks in ((4, [1, 1], 0, 0), (4, [1, 1], 20, 2), (2, [60, 9], 0, 0), (2, [60, 9], 16, 1), (1, [150, 2], 0, 0), (1, [150, 2], 33, 0)):
        b = Batch(7 + group, [160, 75], news, 2, group, 128, 16, dtype)
        for r, j, block in ((0, 0, 1), (0, 120, 3), (0, 131, 0), (1, 30, 2), (1, 74, 0)):
            s = b.slot(r, j)
            b.cache.data[s // 16, 1, 2 * b.cache.codes + which * b.cache.scales + (s % 16) * 4 + block] = 255
        got = b.check(window, sinks)
        assert np.isnan(got).any() and not np.isnan(got[:, :group]).any()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_queries_that_are_not_numbers_stay_among_themselves(gpu_device, dtype):
    for news in ([1, 1, 1], [40, 3, 30]):
        b = Batch(4, [60, 50, 33], news, 2, 4, 64, 32, dtype)
        clean = b.run()
        b.q[1, 2, 7], b.q[-1, 5, 0] = np.nan, np.inf
        got = b.run()
        hit = np.zeros(got.shape[:2], bool)
        hit[1, 2] = hit[-1, 5] = True
        assert np.isnan(got[1, 2]).all() and np.isnan(got[-1, 5]).all() and np.array_equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("scale,strong", [(0.0, 1.0), (-0.3, 1.0), (1.0, 6.0), (0.088, 1e-3), (2.0, 1e-30)])
def test_scales(gpu_device, scale, strong, dtype):
    """Uniform weights, inverted ones, scores of hundreds (one token takes all), scores of nothing."""
    Batch(5, [100, 67, 9], [1, 1, 1], 2, 4, 128, 16, dtype, strong=strong).check(scale=scale)
    Batch(6, [100, 67, 9], [50, 67, 1], 1, 4, 128, 16, dtype, strong=strong).check(scale=scale)


def test_many_requests(gpu_device):
    """More than one trip of 64 over the requests, some without tokens."""
    g = np.random.default_rng(8)
    lengths = g.integers(1, 40, 150).tolist()
    news = [min(n, int(g.integers(0, 3))) for n in lengths]
    lengths[77], news[77] = 300, 40
    Batch(9, lengths, news, 2, 2, 64, 16).check()


def large(seed, lengths, news, kv_heads, group, dim, page, dtype="bf16"):
    """A batch whose cache is made on the GPU, for lengths that the oracle's loops are too slow for; and its pages as numbers."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    pages = sum(need)
    data = torch.randint(0, 256, (pages, kv_heads, page_bytes(page, dim)), dtype=torch.uint8, device="cuda", generator=g)
    data[:, :, page * dim:] = torch.randint(124, 127, (pages, kv_heads, page * dim // 16), dtype=torch.uint8, device="cuda", generator=g)
    ids = torch.randperm(pages, device="cuda", generator=g).int()
    table = torch.full((len(lengths), max(need)), -1, dtype=torch.int32, device="cuda")
    for r, n in enumerate(need):
        table[r, :n] = ids[sum(need[:r]):sum(need[:r]) + n]
    T = sum(news)
    q = torch.randn((T, kv_heads * group, dim), device="cuda", generator=g).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    return data, table, q


def plain(data, table, q, lengths, news, kv_heads, group, dim, page, window, sinks):
    """The definition in 64 bits with torch on the GPU, a request and a head at a time, and what compare() asks for."""
    values = torch.tensor(ref.CODE_VALUES, dtype=torch.float64, device="cuda")
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    v_max, qk, count = (torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda") for _ in range(3))
    t0, half, tail = 0, page * dim // 2, page * dim // 32
    for r, (L, n) in enumerate(zip(lengths, news)):
        raw = data[table[r, :-(-L // page)].long()]
        p, j = torch.arange(L - n, L, device="cuda")[:, None], torch.arange(L, device="cuda")[None, :]
        sees = (j <= p) & ((j > p - window) | (j < sinks)) if window else j <= p
        for h in range(kv_heads):
            def part(which):
                c = raw[:, h, which * half:(which + 1) * half].reshape(-1, dim // 2)[:L]
                s = raw[:, h, 2 * half + which * tail:2 * half + (which + 1) * tail].reshape(-1, dim // 32)[:L].double()
                c = torch.stack((c & 15, c >> 4), -1).reshape(L, dim).long()
                return torch.where(c >= 8, -values[c & 7], values[c & 7]) * (2.0 ** (s - 127)).repeat_interleave(32, -1)
            k, v = part(0), part(1)
            for a in range(h * group, (h + 1) * group):
                x = q[t0:t0 + n, a].double()
                z = (x @ k.t().contiguous()) * dim ** -0.5
                out[t0:t0 + n, a] = torch.softmax(z.masked_fill(~sees, float("-inf")), -1) @ v
                v_max[t0:t0 + n, a] = v.abs().max()
                qk[t0:t0 + n, a] = (x.abs() @ k.abs().t().contiguous()).masked_fill(~sees, 0.0).amax(-1) * dim ** -0.5
                count[t0:t0 + n, a] = sees.sum(-1).double()
        t0 += n
    return out.cpu().numpy(), tuple(x.cpu().numpy() for x in (v_max, qk, count))


@pytest.mark.parametrize("lengths,news,kv_heads,group,dim,page,window,sinks,dtype", [
    ([30001], [1], 2, 4, 128, 64, 0, 0, "bf16"),                      # one request, cut into pieces
    ([30001, 5, 9000], [1, 1, 1], 1, 8, 64, 16, 0, 0, "bf16"),
    ([30001, 12345], [1, 1], 2, 4, 128, 16, 5000, 100, "bf16"),
    ([9001, 4000], [2, 7], 1, 3, 64, 32, 0, 0, "f32"),
    ([20000] * 40, [1] * 40, 4, 2, 64, 256, 0, 0, "bf16"),            # as many as the chip holds workgroups, and more
    ([2100], [2100], 2, 4, 128, 64, 0, 0, "bf16"),                    # a prompt
    ([2500, 700], [1900, 333], 1, 8, 64, 16, 600, 5, "bf16"),
    ([16000], [130], 1, 2, 128, 128, 0, 0, "bf16"),                   # few rows on a long context
    ([9000, 9100], [77, 1], 2, 7, 128, 64, 0, 0, "bf16"),
    ([9000, 300, 9100], [129, 200, 1], 1, 5, 64, 16, 4000, 30, "bf16"),
    ([1030], [1030], 1, 2, 64, 16, 0, 0, "f32"),
])
def test_long(gpu_device, lengths, news, kv_heads, group, dim, page, window, sinks, dtype):
    data, table, q = large(sum(lengths), lengths, news, kv_heads, group, dim, page, dtype)
    T, heads = q.shape[0], q.shape[1]
    kv = P.make_kv_desc(data.shape[0], page, kv_heads, dim, len(lengths), table.shape[1])
    at = P.make_attention_desc(T, heads, dim, dtype, max(news), window, sinks)
    n = P.emoe_kv_attention_workspace_bytes(kv, at)
    cu = torch.tensor(np.concatenate(([0], np.cumsum(news))), dtype=torch.int32, device="cuda")
    seq = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    outs = []
    for fill in (255, 0):  # what the workspace held does not matter, and a second run has the same bits
        ws, out = torch.full((n,), fill, dtype=torch.uint8, device="cuda"), torch.full_like(q, 3.0)
        P.emoe_kv_attention(kv, at, q, data, table, seq, cu, out, ws, n)
        torch.cuda.synchronize()
        outs.append(out)
    assert torch.equal(outs[0], outs[1])
    compare(outs[0].double().cpu().numpy(), *plain(data, table, q, lengths, news, kv_heads, group, dim, page, window, sinks), dim, dtype)


@pytest.mark.parametrize("news", (1, 200))
def test_a_cache_past_four_gigabytes(gpu_device, news):
    """The request's pages lie beyond 4 GiB."""
    heads, dim, page, L = 8, 128, 64, 500
    per_page = heads * page_bytes(page, dim)
    pages = (9 << 29) // per_page
    small, table, q = large(77, [L], [news], heads, 2, dim, page)
    data = torch.zeros((pages, heads, page_bytes(page, dim)), dtype=torch.uint8, device="cuda")
    assert data.numel() > 1 << 32
    data[pages - small.shape[0]:] = small
    moved = table + (pages - small.shape[0])
    kv = P.make_kv_desc(pages, page, heads, dim, 1, table.shape[1])
    at = P.make_attention_desc(news, 2 * heads, dim, "bf16", news)
    n = P.emoe_kv_attention_workspace_bytes(kv, at)
    out, ws = torch.zeros_like(q), torch.empty(n, dtype=torch.uint8, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    P.emoe_kv_attention(kv, at, q, data, moved.int(), torch.tensor([L], **i32), torch.tensor([0, news], **i32), out, ws, n)
    torch.cuda.synchronize()
    compare(out.double().cpu().numpy(), *plain(small, table, q, [L], [news], heads, 2, dim, page, 0, 0), dim, "bf16")


def test_lengths_that_make_no_sense_stay_in_bounds(gpu_device):
    """Offsets that run backwards or beyond T, lengths of 2^31 - 1: whatever comes out, other rows and the memory around stay
    as they are (the buffers of Batch.run are checked there)."""
    b = Batch(11, [64, 100, 40], [2, 3, 1], 2, 4, 64, 16)
    good = b.run()
    b.cu = np.array([0, 2, 5, 1 << 30], dtype=np.int32)
    got = b.run()
    assert np.array_equal(got[:5], good[:5])
    b.cu = np.array([0, 2, -9, 1], dtype=np.int32)
    b.run()
    b.cu = np.array([0, 2, 5, 6], dtype=np.int32)
    b.lengths = [64, (1 << 31) - 1, 40]
    got = b.run()
    assert np.array_equal(got[:2], good[:2]) and np.array_equal(got[5:], good[5:])
    b.lengths = [64, -(1 << 31), 40]
    got = b.run()
    assert np.array_equal(got[:2], good[:2]) and np.array_equal(got[5:], good[5:]) and not got[2:5].any()


@pytest.mark.parametrize("news", ([1, 1], [100, 3]))
def test_another_stream_and_a_graph(gpu_device, news):
    """A whole step (tables, append, attention) on a stream of its own and as a graph that is replayed with other lengths."""
    heads, group, dim, page, R = 2, 4, 64, 16, 2
    T, pages, width = sum(news), 64, 30
    kv = P.make_kv_desc(pages, page, heads, dim, R, width)
    at = P.make_attention_desc(T, heads * group, dim, "bf16", max(news))
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q = torch.randn((T, heads * group, dim), device="cuda", generator=g).bfloat16()
    k, v = (torch.randn((T, heads, dim), device="cuda", generator=g).bfloat16() for _ in range(2))
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = torch.randint(0, 120, (pages, heads, page_bytes(page, dim)), dtype=torch.uint8, device="cuda", generator=g)
    table = torch.full((R, width), -1, **i32)
    table[0, :10], table[1, :10] = torch.arange(10, **i32), torch.arange(10, 20, **i32)  # held; the pages from 20 on are free
    length, new = torch.tensor([40, 17], **i32), torch.tensor(news, **i32)
    ring, c0, c1 = (torch.arange(pages, **i32) + 20) % pages, torch.tensor([0, pages - 20], device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    cu, slot, pos, seq, refused = (torch.zeros(n, **i32) for n in (R + 1, T, T, R, 1))
    n = P.emoe_kv_attention_workspace_bytes(kv, at)
    ws, out = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros_like(q)

    def step(stream=None):
        P.emoe_kv_plan(kv, T, length, new, table, ring, c0, cu, slot, pos, seq, c1, refused, stream)
        P.emoe_kv_append(kv, T, "bf16", k, v, slot, cache, stream=stream)
        P.emoe_kv_attention(kv, at, q, cache, table, seq, cu, out, ws, n, stream)

    fresh = table.clone()
    wants = []
    for l in ([40, 17], [3, 100], [0, 0]):
        length.copy_(torch.tensor(l, **i32))
        table.copy_(fresh)
        before = cache.clone()
        step()
        torch.cuda.synchronize()
        wants.append((l, before, out.clone()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for l, before, want in wants + wants[::-1]:
        for replay in (True, False):
            length.copy_(torch.tensor(l, **i32))
            table.copy_(fresh)
            cache.copy_(before)
            out.fill_(9.0)
            torch.cuda.synchronize()
            graph.replay() if replay else step(side)
            torch.cuda.synchronize()
            assert torch.equal(out, want), (l, replay)


@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 40)])
def test_a_call_that_could_have_more_work_than_31_bits_count(gpu_device, window, sinks):
    """A table of 2^23 tokens, 256 heads and room for 2048 query tokens, of which 23 come."""
    b = Batch(12, [40, 600], [3, 20], 256, 1, 64, 256, "f32")
    wide = np.full((2, 1 << 15), -1, dtype=np.int32)
    wide[:, :b.table.shape[1]] = b.table
    want, seen = ref.attention(b.cache, b.q, b.table, b.lengths, b.cu, 64 ** -0.5, window, sinks)
    b.table, b.T = wide, 2048
    b.q = np.concatenate((b.q, np.zeros((2048 - 23, 256, 64))))
    compare(b.run(window, sinks, max_new=1024)[:23], want, seen, 64, "f32")
