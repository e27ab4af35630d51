"""From one step to the next: the lengths that requests then hold, pages of refused requests that end, and one step captured and replayed as the next ones."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from oracle import kv_cache as ref
from test_gpu_kv_serving import free
from test_gpu_kv_tables import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R", (0, 1, 64, 257, 1000))
@pytest.mark.parametrize("use_ended", (True, False))
def test_lengths(gpu_device, R, use_ended):
    g = np.random.default_rng(R)
    held, seq, ended = g.integers(-1, 100, R), g.integers(-1, 200, R) * g.integers(0, 2, R), g.integers(0, 3, R)
    length = dev(np.append(held, -7))
    P.emoe_kv_advance(P.make_kv_desc(4, 16, 1, 64, R, 1), dev(seq) if R else None, dev(ended) if use_ended and R else None, length)
    torch.cuda.synchronize()
    assert length[R].item() == -7
    assert length[:R].tolist() == ref.advance(held, seq, ended if use_ended else None)


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_a_refused_row_that_ends_gives_its_pages_back(gpu_device, window, sinks):
    """Its length after the step is 0, as the tables' call leaves it: what it held before is what goes back."""
    table = np.array([[0, 1, 2, 3], [4, 5, 6, 7]])
    before, now, ended = [60, 33], [0, 40], [1, 0]
    ring = np.full(12, -9)
    want_ring, want = ref.release(16, before, now, ended, window, sinks, table, ring, (2, 5))
    assert want[1] - 5 >= (3 if window else 4)
    kv = P.make_kv_desc(12, 16, 1, 64, 2, 4)
    f, c, after = dev(ring), dev([2, 5], torch.int64), dev([0, 0], torch.int64)
    P.emoe_kv_release(kv, dev(before), dev(now), dev(ended), window, sinks, dev(table), f, c, after)
    torch.cuda.synchronize()
    assert f.tolist() == want_ring.tolist() and after.tolist() == want


def test_one_captured_step_replays_as_the_next(gpu_device):
    """A graph of one decode step, ten times, against the calls themselves: lengths, tables, ring and outputs go on from step to step."""
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    kvs = [P.KvCache.allocate(1, 3, 100, 14, 16, 2, 64, 128, window=40, sinks=2) for _ in range(2)]
    x = torch.randn((70, 8, 64), generator=g, device="cuda").bfloat16()
    for kv in kvs:
        kv.plan(torch.tensor([60, 3, 7], **i32), 70)
        kv.append(0, x[:, 4:6], x[:, 6:])
        kv.release()
    rows, new, ended = torch.empty((3, 8, 64), device="cuda").bfloat16(), torch.ones(3, **i32), torch.zeros(3, **i32)
    outs = [torch.zeros((3, 4, 64), device="cuda").bfloat16() for _ in range(2)]

    def step(kv, out):
        kv.plan(new, 3)
        kv.append(0, rows[:, 4:6], rows[:, 6:])
        kv.attend(0, rows[:, :4], out, 1)
        kv.release(ended)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(kvs[0], outs[0])
    for n in range(10):
        rows.copy_(torch.randn(rows.shape, generator=g, device="cuda"))
        ended.copy_(torch.tensor([0, n == 4, 0], **i32))
        graph.replay()
        torch.cuda.synchronize()
        step(kvs[1], outs[1])
        (outs[1].float() @ torch.ones(64, device="cuda")).sum().item()
        assert torch.equal(outs[0], outs[1]) and outs[0].any()
        assert kvs[0].length[0].tolist() == kvs[1].length[0].tolist() == [61 + n, (4 + n) if n < 4 else n - 4, 8 + n]
        assert free(kvs[0]) == free(kvs[1]) and torch.equal(kvs[0].block_table, kvs[1].block_table) and kvs[0].refused.item() == 0
