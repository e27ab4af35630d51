"""The cache through its Python class, and the example that serves requests with it next to the MoE layer."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from kv_util import compare
from oracle import kv_cache as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("serve_moe", os.path.join(ROOT, "examples", "serve_moe.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def free(kv):
    head, tail = kv.counters[0].tolist()
    ring = kv.free_pages.tolist()
    return sorted(ring[i % len(ring)] for i in range(head, tail))


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_the_example_serves_all_and_gives_all_pages_back(gpu_device, window, sinks):
    serve_moe = example()
    model = serve_moe.Model()
    prompts = [[1, 2, 3], list(range(40)), [7]]
    made, kv = serve_moe.serve(model, prompts, 12, window, sinks)
    assert [len(m) for m in made] == [12, 11, 10]
    assert free(kv) == list(range(kv.desc.pages)) and kv.length[0].tolist() == [0, 0, 0]
    again, _ = serve_moe.serve(model, prompts, 12, window, sinks)
    assert made == again


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 5)])
def test_steps_of_any_size_attend_alike(gpu_device, window, sinks):
    """The same tokens brought in one step, and a few at a time: every token's output is the oracle's."""
    g = np.random.default_rng(4)
    R, heads, kv_heads, dim, page, total = 3, 6, 2, 64, 16, [90, 33, 61]
    i32 = dict(dtype=torch.int32, device="cuda")
    rows = [torch.from_numpy(g.standard_normal((n, heads + 2 * kv_heads, dim))).bfloat16().cuda() for n in total]
    results = []
    for most in (max(total), 7, 1):
        kv = P.KvCache.allocate(1, R, 96, 24, page, kv_heads, dim, sum(total), window=window, sinks=sinks)
        done, outs = [0] * R, [[] for _ in range(R)]
        step = 0
        while any(d < n for d, n in zip(done, total)):
            new = [min(n - d, max(1, most - (step + r) % 3)) for r, (d, n) in enumerate(zip(done, total))]
            x = torch.cat([rows[r][done[r]:done[r] + new[r]] for r in range(R)])
            kv.plan(torch.tensor(new, **i32), sum(new))
            kv.append(0, x[:, heads:heads + kv_heads], x[:, heads + kv_heads:])
            out = kv.attend(0, x[:, :heads], torch.empty((sum(new), heads, dim), dtype=x.dtype, device="cuda"), max(new))
            assert kv.refused.item() == 0
            at = 0
            for r in range(R):
                outs[r].append(out[at:at + new[r]])
                at += new[r]
                done[r] += new[r]
            kv.release()
            step += 1
        results.append([torch.cat(o).double().cpu().numpy() for o in outs])
        if window:  # what is out of sight has been given back
            kept = [-(-n // page) - (max(-(-sinks // page), (n - window + 1) // page) - -(-sinks // page)) for n in total]
            assert len(free(kv)) == 24 - sum(kept)
    for r, n in enumerate(total):
        x = rows[r].double().cpu().numpy()
        data = np.zeros((-(-n // page), kv_heads, page * dim * 17 // 16), dtype=np.uint8)
        cache = ref.Cache(data, page, dim)
        for j in range(n):
            cache.write(j, 0, *ref.quantise(x[j, heads:heads + kv_heads]))
            cache.write(j, 1, *ref.quantise(x[j, heads + kv_heads:]))
        want, seen = ref.attention(cache, x[:, :heads], np.arange(data.shape[0])[None], [n], [0, n], dim ** -0.5, window, sinks)
        for got in results:
            compare(got[r], want, seen, dim, "bf16")


def test_a_refused_row_keeps_what_it_holds(gpu_device):
    """Three pages for two requests: the second has to wait until the first ends, and goes on from where it was."""
    kv = P.KvCache.allocate(1, 2, 64, 3, 16, 1, 64, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    x = torch.randn((64, 1, 64), device="cuda").bfloat16()

    def step(new, ended=None):
        T = sum(new)
        kv.plan(torch.tensor(new, **i32), T)
        kv.append(0, x[:T], x[:T])
        out = kv.attend(0, x[:T], torch.empty_like(x[:T]), max(new))
        refused = kv.refused.item()
        kv.release(None if ended is None else torch.tensor(ended, **i32))
        return refused, out

    assert step([20, 10])[0] == 0 and kv.length[0].tolist() == [20, 10]
    refused, out = step([2, 10])  # the second would need a page more
    assert refused == 1 and not out[2:].any() and out[:2].any() and kv.length[0].tolist() == [22, 10] and free(kv) == []
    assert step([1, 0], [1, 0])[0] == 0 and kv.length[0].tolist() == [0, 10] and len(free(kv)) == 2
    assert step([0, 10])[0] == 0 and kv.length[0].tolist() == [0, 20]
    with pytest.raises(ValueError):
        kv.plan(torch.tensor([60, 60], **i32), 120)


def test_two_steps_as_a_graph(gpu_device):
    """Two decode steps (the counters and lengths change places) captured once and replayed with other inputs, with work of another kind
    between the replays: the same as the calls themselves."""
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    kvs = [P.KvCache.allocate(2, 4, 200, 40, 16, 2, 128, 256, window=90, sinks=4) for _ in range(2)]
    prompts = [70, 3, 120, 31]
    x = torch.randn((sum(prompts), 12, 128), generator=g, device="cuda").bfloat16()
    for kv in kvs:
        kv.plan(torch.tensor(prompts, **i32), sum(prompts))
        for layer in range(2):
            kv.append(layer, x[:, 8:10], x[:, 10:])
        kv.release()
    rows = torch.empty((2, 4, 12, 128), device="cuda").bfloat16()  # of two steps
    outs = [torch.zeros((2, 2, 4, 8, 128), device="cuda").bfloat16() for _ in range(2)]
    ones, ended = torch.ones(4, **i32), torch.zeros(4, **i32)

    def steps(kv, out):
        for s in range(2):
            kv.plan(ones, 4)
            for layer in range(2):
                kv.append(layer, rows[s, :, 8:10], rows[s, :, 10:])
                kv.attend(layer, rows[s, :, :8], out[s, layer], 1)
            kv.release(ended)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        steps(kvs[0], outs[0])
    for n in range(8):
        rows.copy_(torch.randn(rows.shape, generator=g, device="cuda"))
        ended.copy_(torch.tensor([0, n == 2, 0, n == 5], **i32))
        graph.replay()
        torch.cuda.synchronize()
        steps(kvs[1], outs[1])
        (outs[1].float() @ torch.ones(128, device="cuda")).sum().item()
        assert torch.equal(outs[0], outs[1]) and outs[0].any()
        assert torch.equal(kvs[0].length[0], kvs[1].length[0]) and free(kvs[0]) == free(kvs[1])
        assert torch.equal(kvs[0].block_table, kvs[1].block_table) and kvs[0].refused.item() == 0


def test_a_step_on_another_stream(gpu_device):
    """Everything on a stream that is not the current one, as an object and as its address."""
    i32 = dict(dtype=torch.int32, device="cuda")
    x = torch.randn((30, 3, 64), device="cuda").bfloat16()
    results = []
    for stream in (None, torch.cuda.Stream(), torch.cuda.Stream().cuda_stream):
        kv = P.KvCache.allocate(1, 2, 64, 8, 16, 1, 64, 32)
        new, ended, out = torch.tensor([20, 10], **i32), torch.tensor([0, 1], **i32), torch.empty((30, 1, 64), device="cuda").bfloat16()
        torch.cuda.synchronize()
        kv.plan(new, 30, stream)
        kv.append(0, x[:, 1:2], x[:, 2:], stream)
        kv.attend(0, x[:, :1], out, 20, stream=stream)
        kv.release(ended, stream)
        torch.cuda.synchronize()
        results.append((out, kv.length[0].tolist(), free(kv)))
    assert results[0][1] == [20, 0] and results[0][2] == [2, 3, 4, 5, 6, 7]
    for r in results[1:]:
        assert torch.equal(r[0], results[0][0]) and r[1:] == results[0][1:]
