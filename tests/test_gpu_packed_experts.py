"""The layer's calls with experts in 8 bits against the oracle: the FFN element by element, and what goes with it."""

import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from oracle import packed as ref
from packed_util import HALF_STEP, as_device, close, packed, tokens, weights

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, T, d, f, S, k, act="swiglu", seed=0, sizes=None):
        """Rows are shared out evenly but for an expert without any; `sizes`: rows of each slot, one expert a token."""
        g = np.random.default_rng(seed + T + d)
        self.T, self.d, self.f, self.S, self.k, self.act, self.g = T, d, f, S, k, act, g
        self.x = tokens(g, T, d)
        self.m1, self.m3, self.m2 = (packed([weights(g, a, b) for _ in range(S)]) for a, b in ((f, d), (f, d), (d, f)))
        if act == "relu":
            self.m3 = None
        if sizes is not None:
            self.slots = g.permutation(np.repeat(np.arange(S), sizes))[:, None]
        else:
            free = S - 1 if S > k else S
            self.slots = np.stack([g.permutation(free)[:k] for _ in range(T)])
        flat = self.slots.reshape(-1)
        self.perm = np.argsort(flat, kind="stable")
        self.inverse = np.argsort(self.perm, kind="stable")
        self.offsets = np.concatenate(([0], np.cumsum(np.bincount(flat, minlength=S))))
        self.weight = torch.softmax(torch.from_numpy(g.standard_normal((T, k))), 1).float()
        self.desc = P.make_desc(T, d, f, S, k, S, "f8", act)
        self.ws = torch.full((P.emoe_workspace_bytes(self.desc)[1],), 255, dtype=torch.uint8, device="cuda")
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).int().cuda()
        self.dev = dict(x=as_device(self.x), perm=i32(self.perm), inv=i32(self.inverse), offsets=i32(self.offsets), weight=self.weight.cuda())
        self.y = torch.full((T * k + 1, d), 5.0, dtype=torch.bfloat16, device="cuda")
        self.out = torch.full((T + 1, d), 5.0, dtype=torch.bfloat16, device="cuda")

    def experts(self):
        y, off = np.zeros((self.T * self.k, self.d)), np.zeros((self.T * self.k, self.d))
        m1, m2 = self.m1.cpu().numpy(), self.m2.cpu().numpy()
        m3 = None if self.m3 is None else self.m3.cpu().numpy()
        for s in range(self.S):
            rows = slice(self.offsets[s], self.offsets[s + 1])
            if rows.stop > rows.start:
                y[rows], off[rows] = ref.expert_ffn(self.x[self.perm[rows] // self.k], m1[s], None if m3 is None else m3[s], m2[s], self.f)
        return y, off

    def gather(self, stream=None):
        v = self.dev
        P.emoe_expert_ffn_gather(self.desc, v["x"], v["perm"], v["offsets"], self.m1, self.m3, self.m2, self.y, self.ws, self.ws.numel(), stream)

    def combine(self, stream=None):
        v = self.dev
        P.emoe_expert_ffn_gather_combine(self.desc, v["x"], v["perm"], v["inv"], v["offsets"], self.m1, self.m3, self.m2, v["weight"], self.y, self.out,
                                         self.ws, self.ws.numel(), stream)


CASES = [
    # T, d, f, S, k, act
    (1, 128, 128, 2, 1, "swiglu"), (1, 264, 520, 8, 2, "swiglu"), (5, 8, 8, 3, 2, "swiglu"), (16, 136, 264, 4, 2, "relu"), (40, 264, 392, 4, 2, "swiglu"),
    (64, 512, 1096, 6, 2, "swiglu"), (100, 264, 136, 16, 6, "swiglu"), (130, 392, 264, 2, 1, "relu"), (300, 264, 520, 3, 2, "swiglu"),
    (700, 136, 264, 2, 1, "swiglu"), (600, 264, 392, 2, 2, "relu"), (33, 1032, 1416, 64, 8, "swiglu"),
]


@pytest.mark.parametrize("T,d,f,S,k,act", CASES)
def test_expert_ffn(gpu_device, T, d, f, S, k, act):
    a = Layer(T, d, f, S, k, act)
    want, off = a.experts()
    a.gather()
    torch.cuda.synchronize()
    close(a.y[:-1], want, off)
    rel = np.linalg.norm(a.y[:-1].double().cpu().numpy() - want) / np.linalg.norm(want)
    assert rel < 6e-3  # the bf16 rounding is 1.7e-3, codes of h that fall to the other side 1.2e-3
    assert (a.y[-1] == 5.0).all()
    whole = a.y.clone()
    # the rows grouped beforehand, and the two passes one by one: the same bits
    x_perm = a.dev["x"][a.dev["perm"].long() // k].contiguous()
    a.y.fill_(5.0)
    P.emoe_expert_ffn(a.desc, x_perm, a.dev["offsets"], a.m1, a.m3, a.m2, a.y, a.ws, a.ws.numel())
    torch.cuda.synchronize()
    assert torch.equal(a.y, whole)
    a.y.fill_(5.0)
    for which in (1, 2):
        P.emoe_expert_ffn_gather_pass(a.desc, which, a.dev["x"], a.dev["perm"], a.dev["offsets"], a.m1, a.m3, a.m2, a.y, a.ws, a.ws.numel())
    P.emoe_expert_ffn_gather_pass(a.desc, 2, a.dev["x"], a.dev["perm"], a.dev["offsets"], a.m1, a.m3, a.m2, a.y, a.ws, a.ws.numel())  # h is still there
    torch.cuda.synchronize()
    assert torch.equal(a.y, whole)
    # and with the combine
    a.combine()
    torch.cuda.synchronize()
    y = whole[:-1].double().cpu().numpy()[a.inverse].reshape(T, k, d)
    summed = (y * a.weight.double().numpy()[:, :, None]).sum(1) if k > 1 else y[:, 0]
    close(a.out[:-1], summed, np.abs(y).sum(1) * 2.0 ** -21)
    assert (a.out[-1] == 5.0).all()


@pytest.mark.parametrize("sizes", [(0, 0, 7), (65, 0, 1, 300), (16, 17, 0, 64, 63, 1), (257, 3)])
@pytest.mark.parametrize("act", ("swiglu", "relu"))
def test_uneven_slots(gpu_device, sizes, act):
    a = Layer(sum(sizes), 264, 392, len(sizes), 1, act, sizes=sizes)
    want, off = a.experts()
    a.gather()
    torch.cuda.synchronize()
    close(a.y[:-1], want, off)


@pytest.mark.parametrize("T", (6, 200))
def test_a_nan_token_makes_nan_of_its_own_rows(gpu_device, T):
    a = Layer(T, 264, 392, 4, 2)
    a.dev["x"][3, 200] = float("nan")
    a.dev["x"][T - 1, 7] = float("inf")
    a.combine()
    torch.cuda.synchronize()
    nan = torch.isnan(a.out[:-1])
    assert nan[3].all() and nan[T - 1].all() and int(nan.sum()) == 2 * a.d


@pytest.mark.parametrize("T", (6, 300))
def test_h_beyond_fp32_is_nan_and_large_h_is_not(gpu_device, T):
    """g and u at the edge of fp32: their product passes it, in one row, and only there is the result NaN."""
    a = Layer(T, 136, 264, 1, 1)
    x = np.zeros((T, 136))
    x[:, 0] = 1.0
    x[1, 0] = 2.0 ** 70
    x[2, 0] = 2.0 ** 50
    w = np.zeros((264, 136))
    w[:, 0] = np.linspace(0.5, 1.0, 264)
    m = packed([w.astype(np.float32).astype(np.float64)])
    a.m1 = a.m3 = m
    a.dev["x"] = as_device(x)
    a.combine()
    torch.cuda.synchronize()
    nan = torch.isnan(a.out[:-1])
    assert nan[1].all() and int(nan.sum()) == a.d and torch.isfinite(a.out[2]).all()


def layer_inputs(T, d, f, E, S, k, act="swiglu", seed=1):
    g = np.random.default_rng(seed)
    x = as_device(tokens(g, T, d))
    gate = as_device(weights(g, E, d) * 8)
    m = [packed([weights(g, a, b) for _ in range(E)]) for a, b in ((f, d), (f, d), (d, f))]
    if act == "relu":
        m[1] = None
    slot_of_expert = np.full(E, -1)
    slot_of_expert[g.permutation(E)[:S]] = np.arange(S)
    return x, gate, m, slot_of_expert


@pytest.mark.parametrize("T,d,f,E,S,k,act", [(1, 264, 392, 8, 4, 2, "swiglu"), (50, 264, 392, 8, 5, 2, "swiglu"), (300, 136, 264, 16, 4, 1, "relu"), (700, 264, 136, 8, 4, 2, "swiglu")])
def test_layer_forward_in_one_call_and_in_four(gpu_device, T, d, f, E, S, k, act):
    x, gate, m, soe = layer_inputs(T, d, f, E, S, k, act)
    expert_of_slot = np.argsort(np.where(soe < 0, E, soe))[:S]
    slots = [None if w is None else w[torch.from_numpy(expert_of_slot).cuda()].contiguous() for w in m]
    maps = torch.from_numpy(soe).int().cuda()
    desc = P.make_desc(T, d, f, E, k, S, "f8", act)
    results = []
    for one_call in (False, True):
        b = P.LayerBuffers.allocate(desc)
        P.layer_forward(b, x, gate, None, maps, *slots, one_call=one_call)
        torch.cuda.synchronize()
        results.append([t.clone() for t in (b.topk_expert, b.topk_weight, b.slot_offsets, b.perm, b.inv_perm, b.out)])
    for u, v in zip(*results):
        assert torch.equal(u, v)
    # routing is that of a bf16 layer
    bf = P.make_desc(T, d, f, E, k, S, "bf16", act)
    te, tw = torch.empty_like(results[0][0]), torch.empty_like(results[0][1])
    P.emoe_route(bf, x, gate, None, maps, te, tw)
    torch.cuda.synchronize()
    assert torch.equal(te, results[0][0]) and torch.equal(tw, results[0][1])
    # and the output that of its experts, token by token
    te, tw = te.cpu().numpy(), tw.double().cpu().numpy()
    xs, out = x.double().cpu().numpy(), results[0][-1]
    for t in sorted({0, T // 2, T - 1}):
        y, off = np.zeros(d), np.zeros(d)
        for j in range(k):
            e = te[t, j]
            v, o = ref.expert_ffn(xs[t:t + 1], m[0][e].cpu().numpy(), None if m[1] is None else m[1][e].cpu().numpy(), m[2][e].cpu().numpy(), f)
            y += tw[t, j] * v[0]
            off += tw[t, j] * (o[0] + (np.abs(v[0]) + o[0]) * (HALF_STEP if k > 1 else 0.0) + np.abs(v[0]) * 2.0 ** -21)
        close(out[t:t + 1], y[None], off[None])


def test_graph_replays_with_eager_work_between(gpu_device):
    for T in (9, 400):
        a = Layer(T, 264, 392, 4, 2)
        x0, x1 = a.dev["x"].clone(), as_device(tokens(a.g, T, 264))
        want = []
        for x in (x0, x1):
            a.dev["x"].copy_(x)
            a.combine()
            torch.cuda.synchronize()
            want.append(a.out.clone())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            a.combine()
        for i in (1, 0, 0, 1):
            a.dev["x"].copy_((x0, x1)[i])
            a.out.zero_()
            a.ws.fill_(255 * (i ^ 1))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(a.out[:-1], want[i][:-1])
            a.dev["x"].copy_((x0, x1)[i ^ 1])
            a.combine()
            torch.cuda.synchronize()
            assert torch.equal(a.out[:-1], want[i ^ 1][:-1])


def test_packed_experts_are_loaded(gpu_device):
    """Host masters in 8 bits into the slots, through the load call, and a layer on them."""
    E, S, k, T, d, f = 6, 3, 2, 20, 136, 264
    x, gate, m, _ = layer_inputs(T, d, f, E, S, k)
    host = [w.cpu().pin_memory() for w in m]
    assert host[0][0].numel() == P.emoe_matrix_bytes(f, d) and host[2][0].numel() == P.emoe_matrix_bytes(d, f)
    desc = P.make_desc(T, d, f, E, k, S, "f8", "swiglu")
    slots = [torch.full((S + 1, w.shape[1]), 170, dtype=torch.uint8, device="cuda") for w in m]
    soe, eos = (torch.full((n,), -1, dtype=torch.int32, device="cuda") for n in (E, S))
    mirror = np.full(S, -1, dtype=np.int32)
    side = torch.cuda.Stream()
    done = P.make_event()
    P.emoe_load_experts(desc, [4, 1, 5], [0, 1, 2], *[[h[e] for e in range(E)] for h in host], *slots, soe, eos, mirror, side, None, done)
    torch.cuda.current_stream().wait_event(done)
    b = P.LayerBuffers.allocate(desc)
    P.layer_forward(b, x, gate, None, soe, *[s[:S] for s in slots], one_call=True)
    torch.cuda.synchronize()
    assert mirror.tolist() == [4, 1, 5] and soe.tolist() == [-1, 1, -1, -1, 0, 2]
    for s, w in zip(slots, m):
        assert torch.equal(s[:S], w[[4, 1, 5]]) and (s[S] == 170).all()
    want = P.LayerBuffers.allocate(desc)
    P.layer_forward(want, x, gate, None, soe, *[w[[4, 1, 5]].contiguous() for w in m])
    torch.cuda.synchronize()
    assert torch.equal(b.out, want.out)


@pytest.mark.parametrize("T,k", [(1, 2), (3, 2), (4, 2), (16, 1), (8, 1), (2, 4)])
@pytest.mark.parametrize("d,act", [(2056, "swiglu"), (1024, "relu")])
def test_few_tokens_whose_rows_the_first_product_converts(gpu_device, T, k, d, act):
    a = Layer(T, d, 264, 5, k, act)
    want, off = a.experts()
    a.gather()
    torch.cuda.synchronize()
    close(a.y[:T * k], want, off)
    # the same from rows that the caller has grouped
    y = torch.full_like(a.y, 5.0)
    grouped = a.dev["x"][torch.from_numpy(a.perm // k).cuda()].contiguous()
    P.emoe_expert_ffn(a.desc, grouped, a.dev["offsets"], a.m1, a.m3, a.m2, y, a.ws, a.ws.numel())
    torch.cuda.synchronize()
    assert torch.equal(y, a.y)


@pytest.mark.parametrize("T,d,f,S,k,act", [
    (3000, 392, 520, 4, 2, "swiglu"), (3000, 392, 1160, 4, 2, "relu"), (6000, 392, 520, 3, 1, "swiglu"), (6000, 264, 1032, 2, 1, "relu"),
    (1500, 520, 3208, 2, 2, "swiglu"), (4000, 136, 1032, 6, 2, "swiglu"), (5000, 1032, 136, 8, 1, "swiglu")])
def test_experts_of_many_rows(gpu_device, T, d, f, S, k, act):
    """Products in tiles, both or one of the two; of one expert a token the second writes the tokens' rows."""
    a = Layer(T, d, f, S, k, act)
    want, off = a.experts()
    if k == 1:
        a.combine()
        torch.cuda.synchronize()
        scale = a.weight.double().numpy()[:, :1]
        y, o = want[a.inverse], off[a.inverse]
        close(a.out[:T], y * scale, (o + (np.abs(y) + o) * HALF_STEP) * scale)
        assert (a.out[T:] == 5.0).all()
    a.gather()
    torch.cuda.synchronize()
    close(a.y[:T * k], want, off)
    assert (a.y[T * k:] == 5.0).all()


def test_packed_experts_through_the_periodic_loader(gpu_device):
    """All experts for the first prompts, then the chosen ones, loaded on the loader's stream."""
    E, k, T, d, f = 6, 2, 90, 136, 264
    x, gate, m, _ = layer_inputs(T, d, f, E, E, k)
    host = [[w[e].cpu().pin_memory() for e in range(E)] for w in m]
    desc = P.make_desc(T, d, f, E, k, E, "f8", "swiglu")
    slots = [torch.full(tuple(w.shape), 255, dtype=torch.uint8, device="cuda") for w in m]
    soe, eos = (torch.full((E,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    b, want = P.LayerBuffers.allocate(desc), P.LayerBuffers.allocate(desc)
    torch.cuda.synchronize()
    loader = P.Loader([dict(desc=desc, host_w1=host[0], host_w3=host[1], host_w2=host[2], w1_slots=slots[0], w3_slots=slots[1], w2_slots=slots[2],
                            slot_of_expert=soe, expert_of_slot=eos)], 2)
    for prompt in range(4):
        _, action = loader.next_prompt()
        if action == P.EMOE_PROMPT_PREDICT:
            loader.update([[5, 1, 2]])
        loader.layer_begin(0)
        P.layer_forward(b, x, gate, None, soe, *slots, one_call=True)
        loader.layer_end(0)
        torch.cuda.synchronize()
        here = loader.residents(0)
        assert sorted(e for e in here if e >= 0) == (list(range(E)) if prompt < 2 else [1, 2, 5])
        own = torch.full((E,), -1, dtype=torch.int32)
        for s, e in enumerate(here):
            if e >= 0:
                own[e] = s
                assert all(torch.equal(a[s], w[e]) for a, w in zip(slots, m))
        resident = [w[[max(e, 0) for e in here]].contiguous() for w in m]
        P.layer_forward(want, x, gate, None, own.cuda(), *resident)
        torch.cuda.synchronize()
        assert torch.equal(b.out, want.out)
    loader.synchronize()
    loader.close()
