"""Matrices in 8 bits through their Python class, alone and as the projections and experts around attention over the cache."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from oracle import packed as ref
from packed_util import as_device, close, numbers, tokens, weights
from test_gpu_kv_serving import example, free

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("count", (1, 3))
def test_matrices_are_packed_and_read_back(gpu_device, dtype, count):
    g = np.random.default_rng(count)
    w = np.stack([weights(g, 136, 264) for _ in range(count)])
    wide = torch.zeros((count, 136, 280), dtype=dtype, device="cuda")
    wide[:, :, 8:272] = torch.from_numpy(w).to("cuda", dtype)
    m = P.PackedMatrices.pack(wide[:, :, 8:272])
    for i in range(count):
        assert np.array_equal(m.data[i].cpu().numpy(), ref.pack(w[i]))
    back = m.read(torch.zeros((count, 136, 264), dtype=dtype, device="cuda"))
    assert np.array_equal(back.double().cpu().numpy(), np.stack(numbers(m.data, 136, 264)))
    again = P.PackedMatrices.allocate(count, 136, 264)
    again.write(back)
    assert torch.equal(again.read(torch.zeros_like(back)), back)


def expected(x, m, i=0):
    """(products with the numbers that the i-th matrix holds, bound of their error) of rows on the device."""
    x = x.double().cpu().numpy()
    q = ref.quantise_rows(x)
    w = numbers(m.data[i:i + 1], m.N, m.K)[0]
    return q @ w.T, ref.product_error(q, ref.rows_least(x), w, ref.matrix_least(m.data[i].cpu().numpy(), m.N, m.K))


@pytest.mark.parametrize("rows", (3, 200))
def test_products_of_slices(gpu_device, rows):
    g = np.random.default_rng(rows)
    m = P.PackedMatrices.pack(as_device(weights(g, 264, 392)))
    x, out = torch.full((rows, 408), 3.0, **{"dtype": torch.bfloat16, "device": "cuda"}), torch.full((rows, 288), 5.0, dtype=torch.bfloat16, device="cuda")
    x[:, 16:] = as_device(tokens(g, rows, 392))
    m.matmul(x[:, 16:], out[:, 16:280], m.workspace(rows))
    assert (out[:, :16] == 5.0).all() and (out[:, 280:] == 5.0).all()
    close(out[:, 16:280], *expected(x[:, 16:], m))


def test_one_workspace_for_products_of_all_sizes_on_a_stream(gpu_device):
    """What a workspace held for one size does not show at another."""
    g = np.random.default_rng(3)
    m = P.PackedMatrices.pack(as_device(weights(g, 136, 520)))
    x = as_device(tokens(g, 300, 520))
    ws = m.workspace(300)
    for rows in (300, 1, 200, 17, 129, 64, 300, 2):
        out = m.matmul(x[:rows], torch.empty((rows, 136), dtype=torch.bfloat16, device="cuda"), ws)
        alone = m.matmul(x[:rows], torch.empty_like(out), m.workspace(rows))
        assert torch.equal(out, alone)
        close(out, *expected(x[:rows], m))


class Step:
    """One layer of a model: projections, attention over the cache, and experts, all matrices in 8 bits."""

    def __init__(self, R, seed, d=264, heads=4, kv_heads=2, dim=64, f=392, E=6, S=4):
        g = np.random.default_rng(seed)
        self.g, self.R, self.d, self.heads, self.kv_heads, self.dim = g, R, d, heads, kv_heads, dim
        pack = lambda *w: P.PackedMatrices.pack(as_device(np.stack(w)))
        self.qkv, self.o = pack(weights(g, (heads + 2 * kv_heads) * dim, d)), pack(weights(g, d, heads * dim))
        self.experts = [pack(*[weights(g, a, b) for _ in range(S)]) for a, b in ((f, d), (f, d), (d, f))]
        self.gate = as_device(weights(g, E, d))
        self.slots = torch.tensor([0, -1, 1, 2, -1, 3], dtype=torch.int32, device="cuda")
        self.layer = P.LayerBuffers.allocate(P.make_desc(R, d, f, E, 2, S, "f8", "swiglu"))
        self.ws = torch.empty(max(self.qkv.workspace_bytes(R), self.o.workspace_bytes(R)), dtype=torch.uint8, device="cuda")
        row = lambda n: torch.empty((R, n), dtype=torch.bfloat16, device="cuda")
        self.projected, self.attended, self.mixed, self.x = row(self.qkv.N), row(heads * dim), row(d), row(d)

    def run(self, kv, new):
        h, k = self.heads, self.kv_heads
        kv.plan(new, self.R)
        self.qkv.matmul(self.x, self.projected, self.ws)
        rows = self.projected.view(self.R, h + 2 * k, self.dim)
        kv.append(0, rows[:, h:h + k], rows[:, h + k:])
        kv.attend(0, rows[:, :h], self.attended.view(self.R, h, self.dim), 1)
        self.o.matmul(self.attended, self.mixed, self.ws)
        out = P.layer_forward(self.layer, self.mixed, self.gate, None, self.slots, *[m.data for m in self.experts], one_call=True)
        kv.release()
        return out

    def check(self, out):
        """The products of the last step, from what the GPU gave them."""
        close(self.projected, *expected(self.x, self.qkv))
        close(self.mixed, *expected(self.attended, self.o))
        b, x = self.layer, self.mixed.double().cpu().numpy()
        perm, offsets = b.perm.cpu().numpy(), b.slot_offsets.cpu().numpy()
        m1, m3, m2 = (m.data.cpu().numpy() for m in self.experts)
        assert offsets[-1] == 2 * self.R
        for s in range(len(offsets) - 1):
            rows = slice(offsets[s], offsets[s + 1])
            if rows.stop > rows.start:
                close(b.y_perm[rows], *ref.expert_ffn(x[perm[rows] // 2], m1[s], m3[s], m2[s], self.experts[0].N))
        # the combine's sum of two bf16 rows in fp32 is rounded once
        y, w = b.y_perm.double().cpu().numpy()[b.inv_perm.cpu().numpy()].reshape(self.R, 2, -1), b.topk_weight.double().cpu().numpy()
        want = (y * w[:, :, None]).sum(1)
        close(out, want, 3 * 2.0 ** -24 * (np.abs(y) * w[:, :, None]).sum(1))


@pytest.mark.parametrize("R", (1, 7, 140))
def test_a_decode_step_of_projections_attention_and_experts(gpu_device, R):
    """Eager steps, each product checked; then the step captured and replayed, against eager ones of the same tokens."""
    step = Step(R, R)
    caches = [P.KvCache.allocate(1, R, 32, 2 * R, 16, step.kv_heads, step.dim, R) for _ in range(2)]
    new = torch.ones(R, dtype=torch.int32, device="cuda")
    inputs = [as_device(tokens(step.g, R, step.d)) for _ in range(5)]
    want = []
    for i, x in enumerate(inputs):
        step.x.copy_(x)
        want.append(step.run(caches[0], new).clone())
        if i in (0, 4):
            step.check(want[-1])
    step.x.copy_(inputs[0])
    assert torch.equal(step.run(caches[1], new), want[0])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        out = step.run(caches[1], new)
    for x, w in zip(inputs[1:], want[1:]):
        step.x.copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, w)


def test_the_example_serves_with_packed_matrices(gpu_device):
    serve_moe = example()
    model = serve_moe.Model(packed=True)
    prompts = [[1, 2, 3], list(range(40)), [7]]
    made, kv = serve_moe.serve(model, prompts, 12)
    assert [len(m) for m in made] == [12, 11, 10]
    assert free(kv) == list(range(kv.desc.pages))
    assert serve_moe.serve(model, prompts, 12)[0] == made
