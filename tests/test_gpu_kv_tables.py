"""emoe_kv_plan and emoe_kv_release against the oracle, every integer of every output."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from oracle import kv_cache as ref

pytestmark = pytest.mark.gpu


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def plan(page, width, T, length, new, table, ring, counters):
    """emoe_kv_plan twice on the same buffers (the second call must not differ), as a dict like the oracle's."""
    R = len(length)
    kv = P.make_kv_desc(len(ring), page, 1, 64, R, width)
    full = lambda n, t=torch.int32: torch.full((n,), -77, dtype=t, device="cuda")
    t, f, c = dev(table), dev(ring), dev(counters, torch.int64)
    cu, slot, pos, seq, after, refused = full(R + 1), full(T + 1), full(T + 1), full(max(R, 1)), full(2, torch.int64), full(1)
    for _ in range(2):
        P.emoe_kv_plan(kv, T, dev(length) if R else None, dev(new) if R else None, t, f, c, cu, slot, pos, seq, after, refused)
        torch.cuda.synchronize()
    assert slot[T] == -77 and pos[T] == -77
    return dict(table=t.cpu().numpy(), cu=cu.tolist(), slot=slot[:T].tolist(), position=pos[:T].tolist(), seq_len=seq[:R].tolist(),
                counters=after.tolist(), refused=refused.item())


def same(got, want):
    for k in want:
        assert np.array_equal(np.asarray(got[k]), np.asarray(want[k])), k


def state(seed, R, page, most, most_new, free, extra=0, head=0):
    """Requests of 0 .. most tokens, new ones from none on, and a ring with `free` pages left of those that they leave."""
    g = np.random.default_rng(seed)
    length, new = g.integers(0, most + 1, R), g.integers(0, most_new + 1, R)
    held = -(-length // page)
    width = int((-(-(length + new) // page)).max(initial=1)) + extra
    pages = int(held.sum()) + max(free, 1)
    ids = g.permutation(pages)
    table = np.full((max(R, 1), max(width, 1)), -1)
    at = 0
    for r in range(R):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    ring = np.full(pages, -5)
    for i in range(free):
        ring[(head + i) % pages] = ids[at + i]
    return length, new, table, ring, (head, head + free)


@pytest.mark.parametrize("seed,R,page,most,most_new,free,T_more,head", [
    (1, 1, 16, 0, 1, 1, 0, 0), (2, 3, 16, 40, 1, 9, 0, 5), (3, 64, 64, 500, 1, 64, 0, (1 << 40) + 3), (4, 70, 16, 100, 33, 400, 7, 11),
    (5, 1025, 32, 90, 3, 1500, 0, 123456789), (6, 2100, 128, 300, 1, 2100, 1, 0), (7, 5, 256, 3000, 900, 40, 0, 77),
    (8, 9, 16, 10, 2500, 2000, 30, 1),                       # rows of several workgroups' tokens
    (9, 40, 16, 30, 20, 10, 0, 2), (10, 1500, 16, 50, 4, 300, 0, 9),  # too few pages
    (11, 30, 16, 30, 20, 0, 0, 2),                           # none
])
def test_plan(gpu_device, seed, R, page, most, most_new, free, T_more, head):
    length, new, table, ring, counters = state(seed, R, page, most, most_new, free, head=head)
    args = (page, table.shape[1], int(new.sum()) + T_more, length, new, table, ring, counters)
    same(plan(*args), ref.plan(*args))


def test_plan_refuses_rows_that_do_not_fit(gpu_device):
    """Rows too long for the table, rows whose tokens end beyond T, negative lengths and counts (none), a table entry of nobody."""
    length, new = [31, 40, -3, 16, 0, 5], [1, 30, 20, -4, 17, 40]
    table = np.array([[0, 1, -1], [2, 3, 4], [-1] * 3, [5, -1, -1], [-1] * 3, [-1, -1, -1]])
    ring = np.array([6, 7, 8, 9, 10, 11, 12, 13])
    ring = np.concatenate((ring, np.arange(14, 30)))
    for T in (108, 107, 60, 51, 21, 1, 0):
        args = (16, 3, T, length, new, table, ring, (0, 24))
        same(plan(*args), ref.plan(*args))


def test_plan_of_nothing(gpu_device):
    for R, T in ((0, 0), (0, 5), (4, 0), (4, 3)):
        args = (16, 2, T, [5] * R, [0] * R, np.full((max(R, 1), 2), 3), np.arange(8), (2, 6))
        same(plan(*args), ref.plan(*args))


@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 9), (1, 0), (17, 0), (17, 1), (64, 4), (100, 16), (33, 200), (5000, 3)])
@pytest.mark.parametrize("seed,R,page,most,grow", [(1, 1, 16, 300, 5), (2, 37, 16, 400, 40), (3, 20, 64, 700, 300), (4, 1030, 32, 200, 90)])
def test_release(gpu_device, window, sinks, seed, R, page, most, grow):
    g = np.random.default_rng(seed + 100 * window)
    before = g.integers(0, most + 1, R)
    now = before + g.integers(0, grow + 1, R)
    ended = g.integers(0, 3, R) == 0
    held = -(-now // page)
    pages = int(held.sum()) + 3
    width = int(held.max()) + 1
    table = np.full((R, width), -1)
    ids, at = g.permutation(pages), 0
    for r in range(R):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    for use_ended in (True, False):
        tail = int(g.integers(0, 1 << 45))
        ring = np.full(pages, -9)
        want_ring, want = ref.release(page, before, now, ended if use_ended else None, window, sinks, table, ring, (tail - 2, tail))
        kv = P.make_kv_desc(pages, page, 1, 64, R, width)
        f, c, after = dev(ring), dev([tail - 2, tail], torch.int64), dev([0, 0], torch.int64)
        for _ in range(2):  # reads nothing that it writes
            P.emoe_kv_release(kv, dev(before) if window else None, dev(now), dev(ended) if use_ended else None, window, sinks, dev(table), f, c, after)
            torch.cuda.synchronize()
        assert np.array_equal(f.cpu().numpy(), want_ring) and after.tolist() == want


def test_release_without_rows(gpu_device):
    kv = P.make_kv_desc(4, 16, 1, 64, 0, 1)
    f, c, after = dev([1, 2, 3, 4]), dev([5, 7], torch.int64), dev([0, 0], torch.int64)
    P.emoe_kv_release(kv, None, None, None, 0, 0, None, f, c, after)
    torch.cuda.synchronize()
    assert f.tolist() == [1, 2, 3, 4] and after.tolist() == [5, 7]


def test_pages_go_round(gpu_device):
    """Twenty steps of four requests that come, grow past a window and end, planned and released in turn with the two pairs of
    counters: no page is ever held twice, none is lost, and the ring's bookkeeping is the oracle's."""
    page, width, pages, R, window, sinks = 16, 12, 40, 4, 48, 5
    g = np.random.default_rng(5)
    kv = P.make_kv_desc(pages, page, 1, 64, R, width)
    table, ring = np.full((R, width), -1), np.arange(pages)
    t, f = dev(table), dev(ring)
    a, b = dev([0, pages], torch.int64), dev([0, 0], torch.int64)
    counters, before, length = (0, pages), np.zeros(R, int), np.zeros(R, int)
    for step in range(20):
        new = g.integers(0, 25, R)
        T = int(new.sum())
        out = {n: torch.zeros(max(k, 1), dtype=torch.int32, device="cuda") for n, k in (("cu", R + 1), ("slot", T), ("pos", T), ("seq", R), ("ref", 1))}
        P.emoe_kv_plan(kv, T, dev(length), dev(new), t, f, a, out["cu"], out["slot"], out["pos"], out["seq"], b, out["ref"])
        want = ref.plan(page, width, T, length, new, table, ring, counters)
        torch.cuda.synchronize()
        assert np.array_equal(t.cpu().numpy(), want["table"]) and b.tolist() == want["counters"] and out["slot"][:T].tolist() == want["slot"]
        assert want["refused"] == 0
        table, counters = want["table"], want["counters"]
        grown = np.array(want["seq_len"])
        ended = (grown > 150) | (g.integers(0, 9, R) == 0)
        P.emoe_kv_release(kv, dev(before), dev(grown), dev(ended), window, sinks, t, f, b, a)
        ring, counters = ref.release(page, before, grown, ended, window, sinks, table, ring, counters)
        torch.cuda.synchronize()
        assert np.array_equal(f.cpu().numpy(), ring) and a.tolist() == counters
        free = [ring[i % pages] for i in range(counters[0], counters[1])]
        assert len(set(free)) == len(free) <= pages
        before, length = np.where(ended, 0, grown), np.where(ended, 0, grown)
