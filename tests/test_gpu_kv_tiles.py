"""emoe_kv_attention's kernel for many queries: requests of more than 512 rows (query tokens times heads on a kv head) go to it whatever
the work is.  As test_gpu_kv_attention, element by element against the oracle."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from kv_util import Batch, compare
from oracle import kv_cache as ref

pytestmark = pytest.mark.gpu

SHAPES = [(1, 40, 128, 16), (2, 47, 64, 64), (1, 64, 128, 256), (1, 33, 64, 16)]  # kv heads, group, dim, page


@pytest.mark.parametrize("kv_heads,group,dim,page", SHAPES)
@pytest.mark.parametrize("lengths,news", [([16], [16]), ([17], [17]), ([70], [20]), ([200], [17]), ([90, 33], [31, 1]), ([64, 129, 20], [16, 16, 16])])
def test_prompts_and_pieces_of_them(gpu_device, kv_heads, group, dim, page, lengths, news):
    Batch(len(lengths) + sum(news) + dim, lengths, news, kv_heads, group, dim, page).check(gap=16)


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32)])
def test_a_token_a_row(gpu_device, dim, page):
    """One query head: 520 tokens, row tiles that begin at tokens 0, 128, 256 and 384."""
    Batch(dim, [520], [520], 1, 1, dim, page).check()
    Batch(dim + 1, [700], [515], 1, 1, dim, page).check(100, 7)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 40), (16, 0), (33, 4), (63, 64), (64, 1), (65, 70), (150, 0), (1000, 7)])
def test_window_and_sinks(gpu_device, window, sinks):
    Batch(window + sinks, [300, 90], [20, 17], 1, 36, 64, 16).check(window, sinks)
    Batch(window + sinks + 1, [260], [30], 1, 20, 128, 64).check(window, sinks)


def test_rows_that_see_nothing_are_zero(gpu_device):
    b = Batch(1, [0, 4, 40, -5], [16, 20, 17, 18], 1, 40, 64, 16)
    b.table[2, :] = -1
    got = b.check()
    cu = b.cu
    assert not got[cu[0]:cu[1]].any() and not got[cu[1]:cu[1] + 16].any() and not got[cu[2]:].any() and got[cu[1] + 16:cu[2]].any()


@pytest.mark.parametrize("dim", (64, 128))
def test_pages_of_nobody_and_lengths_beyond_the_table(gpu_device, dim):
    b = Batch(2, [200, 130], [17, 40], 1, 32, dim, 16)
    b.table[0, 2], b.table[0, 7], b.table[1, 0], b.table[1, 3] = -1, 1 << 30, -7, b.data.shape[0]
    b.check()
    b.check(20, 3)
    b = Batch(3, [300], [20], 1, 32, dim, 16)
    b.table = np.ascontiguousarray(b.table[:, :9])
    full = b.table.copy()
    got = b.run()
    b.table = np.concatenate((full, np.full((1, 12), -1, np.int32)), 1)
    want, seen = ref.attention(b.cache, b.q, b.table, b.lengths, b.cu, dim ** -0.5)
    compare(got, want, seen, dim, "bf16")


@pytest.mark.parametrize("dim", (64, 128))
@pytest.mark.parametrize("which", (0, 1))
@pytest.mark.parametrize("window,sinks", [(0, 0), (16, 1), (33, 0), (0, 5)])
def test_what_is_not_a_number_reaches_those_who_see_it_only(gpu_device, which, dim, window, sinks):
    for group, news in ((40, [60, 16]), (1, [150, 140])):
        if group == 1:
            news, lengths = [530, 3], [560, 75]
        else:
            lengths = [160, 75]
        b = Batch(7 + group, lengths, news, 2, group, dim, 16)
        for r, j, block in ((0, 0, 1), (0, 120, dim // 32 - 1), (0, 131, 0), (1, 30, 1), (1, 74, 0)):
            s = b.slot(r, j)
            b.cache.data[s // 16, 1, 2 * b.cache.codes + which * b.cache.scales + (s % 16) * (dim // 32) + block] = 255
        got = b.check(window, sinks)
        assert np.isnan(got).any() and not np.isnan(got[:, :group]).any()


def test_queries_that_are_not_numbers_stay_among_themselves(gpu_device):
    b = Batch(4, [60, 50], [17, 20], 1, 40, 64, 32)
    clean = b.run()
    b.q[1, 2, 7], b.q[-1, 5, 0] = np.nan, -np.inf
    got = b.run()
    hit = np.zeros(got.shape[:2], bool)
    hit[1, 2] = hit[-1, 5] = True
    assert np.isnan(got[1, 2]).all() and np.isnan(got[-1, 5]).all() and np.array_equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("scale,strong", [(0.0, 1.0), (-0.3, 1.0), (1.0, 6.0), (0.088, 1e-3), (2.0, 1e-30), (1e-30, 1.0)])
@pytest.mark.parametrize("dim", (64, 128))
def test_scales(gpu_device, scale, strong, dim):
    Batch(6, [100, 67], [20, 17], 1, 32, dim, 16, strong=strong).check(scale=scale)


@pytest.mark.parametrize("dim", (64, 128))
def test_scores_that_rise_out_of_range(gpu_device, dim):
    """Keys whose scores grow from tile to tile by hundreds: the weights that the first tile's maximum gives overflow again and
    again.  Then scores that fall as fast, and a row whose first tokens are not seen."""
    for order in (1, -1):
        b = Batch(9, [330], [17], 1, 32, dim, 16)
        for j in range(330):
            s = b.slot(0, j)
            codes = np.zeros((1, dim), dtype=np.uint8)
            codes[0, 0] = 7  # 6 * 2^k along the first axis
            up = j if order > 0 else 329 - j
            b.cache.write(s, 0, codes, np.full((1, dim // 32), 120 + up // 33, dtype=np.uint8))
        b.q[:, :, 0] = np.abs(b.q[:, :, 0]) + 1.0
        b.check(scale=1.0)
        b.check(100, 3, scale=1.0)


def test_a_row_tile_of_every_piece_count(gpu_device):
    """Few row tiles on long contexts: cut into two to many pieces, some of them empty; twice the same bits, with other contents of the
    workspace."""
    from test_gpu_kv_attention import large, plain
    for lengths, news, kv_heads, group, dim, page, window, sinks in (
            ([5000], [520], 1, 1, 64, 64, 0, 0), ([9000], [520], 2, 2, 128, 16, 0, 0), ([4000, 900], [300, 700], 1, 3, 64, 32, 0, 0),
            ([12000], [130], 1, 8, 128, 128, 3000, 50), ([2000, 8000, 100], [600, 515, 1], 1, 1, 128, 64, 0, 0)):
        data, table, q = large(sum(lengths), lengths, news, kv_heads, group, dim, page)
        kv = P.make_kv_desc(data.shape[0], page, kv_heads, dim, len(lengths), table.shape[1])
        at = P.make_attention_desc(q.shape[0], q.shape[1], dim, "bf16", max(news), window, sinks)
        n = P.emoe_kv_attention_workspace_bytes(kv, at)
        cu = torch.tensor(np.concatenate(([0], np.cumsum(news))), dtype=torch.int32, device="cuda")
        seq = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        outs = []
        for fill in (255, 0):
            ws, out = torch.full((n,), fill, dtype=torch.uint8, device="cuda"), torch.full_like(q, 3.0)
            P.emoe_kv_attention(kv, at, q, data, table, seq, cu, out, ws, n)
            torch.cuda.synchronize()
            outs.append(out)
        assert torch.equal(outs[0], outs[1])
        compare(outs[0].double().cpu().numpy(), *plain(data, table, q, lengths, news, kv_heads, group, dim, page, window, sinks), dim, "bf16")


@pytest.mark.parametrize("group", (1, 40))
def test_offsets_that_are_none_reach_no_other_memory(gpu_device, group):
    """Offsets that fall, overlap or lie outside: every request takes what lies between its two within 0 .. T, and nothing else is
    written (Batch.run checks the rows after the last).  A request that stands alone gets what it gets otherwise."""
    b = Batch(5, [600, 90, 70], [520, 20, 16], 1, group, 64, 16)
    good, whole = b.cu.copy(), b.run()
    for cu in ([0, 520, 300, 556], [-5, 520, 1 << 30, 7], [556, 0, -(1 << 31), 520], [0, 556, 0, 556]):
        b.cu = np.array(cu, dtype=np.int32)
        got = b.run(max_new=556)
        if cu[1] == 520 and cu[0] <= 0 and cu[2] != 300:
            assert np.array_equal(got[:520], whole[:520])
    b.cu = good
    assert np.array_equal(b.run(max_new=556), whole)


def _batches():
    """Requests with rows for this kernel among up to 64 and among more; more than 64 of them; more row tiles than places, one request
    far longer than the others, which is cut."""
    g = np.random.default_rng(8)
    few = [int(n) for n in g.integers(1, 400, 130)]
    some = [520 if r in (3, 64, 65, 100, 129) else 1 for r in range(130)]
    yield "five of 130", [n + m for n, m in zip(few, some)], some, 1, 2, 64, 16
    yield "70 of 70", [int(n) for n in g.integers(40, 500, 70)], [40] * 70, 1, 16, 64, 16
    yield "90 of 200", [int(n) for n in g.integers(40, 300, 200)], [40 if r % 20 < 9 else 1 for r in range(200)], 2, 16, 64, 32
    yield "four of 512", [612, 4600, 812, 1500], [512] * 4, 8, 4, 128, 64
    yield "eight, rising", [530 + 300 * r for r in range(8)], [520] * 8, 2, 2, 128, 16


@pytest.mark.parametrize("name,lengths,news,kv_heads,group,dim,page", list(_batches()), ids=lambda v: v.replace(" ", "-") if isinstance(v, str) else "")
def test_batches(gpu_device, name, lengths, news, kv_heads, group, dim, page):
    from test_gpu_kv_attention import large, plain
    data, table, q = large(len(lengths), lengths, news, kv_heads, group, dim, page)
    kv = P.make_kv_desc(data.shape[0], page, kv_heads, dim, len(lengths), table.shape[1])
    at = P.make_attention_desc(q.shape[0], q.shape[1], dim, "bf16", max(news))
    n = P.emoe_kv_attention_workspace_bytes(kv, at)
    ws, out = torch.full((n,), 255, dtype=torch.uint8, device="cuda"), torch.full_like(q, 3.0)
    cu = torch.tensor(np.concatenate(([0], np.cumsum(news))), dtype=torch.int32, device="cuda")
    P.emoe_kv_attention(kv, at, q, data, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), cu, out, ws, n)
    torch.cuda.synchronize()
    compare(out.double().cpu().numpy(), *plain(data, table, q, lengths, news, kv_heads, group, dim, page, 0, 0), dim, "bf16")


def test_pages_beyond_four_gib(gpu_device):
    """A request whose pages are the last of a cache of more than 4 GiB, the same request's in a small one: the same bits."""
    from test_gpu_kv_attention import large
    lengths, news, page, dim = [700], [530], 256, 128
    data, table, q = large(3, lengths, news, 1, 1, dim, page)
    small = data.shape[0]
    pages = (1 << 32) // data[0].numel() + 9
    far = torch.empty((pages, *data.shape[1:]), dtype=torch.uint8, device="cuda")
    far[-small:] = data
    outs = []
    for cache, at_table in ((data, table), (far, table + (pages - small))):
        kv = P.make_kv_desc(cache.shape[0], page, 1, dim, 1, table.shape[1])
        at = P.make_attention_desc(530, 1, dim, "bf16", 530)
        n = P.emoe_kv_attention_workspace_bytes(kv, at)
        ws, out = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
        i32 = dict(dtype=torch.int32, device="cuda")
        P.emoe_kv_attention(kv, at, q, cache, at_table.contiguous(), torch.tensor(lengths, **i32), torch.tensor([0, 530], **i32), out, ws, n)
        torch.cuda.synchronize()
        outs.append(out)
    assert far.numel() > 1 << 32 and torch.equal(*outs) and outs[0].any()


@pytest.mark.parametrize("dim", (64, 128))
def test_large_values_under_rising_scores(gpu_device, dim):
    """Values near 2^88 while the weights climb towards where the maximum is looked for again: fp32 has room for both."""
    b = Batch(10, [330], [17], 1, 32, dim, 16)
    for j in range(330):
        s = b.slot(0, j)
        codes = np.zeros((1, dim), dtype=np.uint8)
        codes[0, 0] = 4  # 2 * 2^k along the first axis
        b.cache.write(s, 0, codes, np.full((1, dim // 32), 127 + j // 110, dtype=np.uint8))
        b.cache.write(s, 1, np.full((1, dim), 6 + 8 * (j % 2), dtype=np.uint8), np.full((1, dim // 32), 127 + 85, dtype=np.uint8))
    b.q[:, :, 0] = 3.0
    got = b.check(scale=1.0)
    assert np.isfinite(got).all() and np.abs(got).max() > 2.0 ** 80
