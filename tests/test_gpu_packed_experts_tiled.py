"""Experts in 8 bits whose products run in tiles, against the oracle: rows grouped beforehand and gathered, single passes, the combine, uneven and empty
slots, NaN, infinities and h beyond fp32, captured calls, repeats and the whole layer, with K cut into pieces and not, in one round of tiles and in more.
Every test says which products it wants in tiles and asks whether they are."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
import test_gpu_packed_experts as streamed
from packed_paths import CUT_FROM, SHORT, blocks, experts_take_tiles
from packed_util import HALF_STEP, as_device, close, packed, tokens

pytestmark = pytest.mark.gpu

COMPUTE_UNITS = 256


def tiles(rows, S, N, swiglu):
    """Output tiles of a product of `rows` rows spread evenly over S groups."""
    return S * -(-(rows // S) // 256) * (blocks(N) if swiglu else -(-blocks(N) // 2))


# T, d, f, S, k, act, products in tiles
CASES = [
    (3100, 264, 1032, 1, 1, "swiglu", (True, False)), (3100, 264, 1160, 2, 2, "relu", (True, False)), (1200, 520, 136, 8, 6, "swiglu", (False, True)),
    (3000, 392, 2056, 3, 2, "relu", (True, True)), (1500, 648, 1416, 8, 4, "swiglu", (True, True)),
    # rows of h of up to five blocks
    (5300, 264, 520, 1, 1, "swiglu", (True, False)), (8300, 392, 264, 2, 1, "relu", (True, True)),
    # more than a round of tiles, of an odd number of blocks of columns
    (6000, 520, 1160, 2, 2, "swiglu", (True, True)), (9000, 392, 2184, 1, 1, "relu", (True, True)),
    # cut along K: the first product, the second, both; behind a round of whole tiles
    (4300, 3208, 520, 1, 1, "swiglu", (True, True)), (2800, 3208, 520, 3, 2, "relu", (True, True)), (2300, 3208, 648, 3, 2, "relu", (True, True)),
    (1500, 648, 3336, 2, 2, "swiglu", (True, True)), (1100, 3336, 3208, 2, 1, "relu", (True, True)), (2100, 3208, 2184, 2, 2, "swiglu", (True, True)),
    (1100, 3208, 3336, 2, 2, "swiglu", (True, True)), (2600, 392, 3208, 2, 2, "relu", (True, True)),
]


@pytest.mark.parametrize("T,d,f,S,k,act,in_tiles", CASES)
def test_every_way_to_call_the_ffn(gpu_device, T, d, f, S, k, act, in_tiles):
    assert experts_take_tiles(T, d, f, S, k) == in_tiles
    streamed.test_expert_ffn(gpu_device, T, d, f, S, k, act)


def test_the_cases_are_of_every_kind():
    cut, rounds = set(), set()
    for T, d, f, S, k, act, in_tiles in CASES:
        here = S - 1 if S > k else S  # (one expert has no rows)
        for i, (tiled, N, K, swiglu) in enumerate(((in_tiles[0], f, d, act == "swiglu"), (in_tiles[1], d, f, False))):
            if tiled:
                n = tiles(T * k, here, N, swiglu)
                cut.add((i, act, i == 0 and blocks(f) <= SHORT, blocks(K) >= CUT_FROM and n % COMPUTE_UNITS <= COMPUTE_UNITS // 2))
                rounds.add((n > COMPUTE_UNITS, blocks(K) % 2, blocks(K) >= CUT_FROM))
    assert cut == {(i, act, short, c) for i, short in ((0, True), (0, False), (1, False)) for act in ("swiglu", "relu") for c in (True, False)}
    assert {(True, 1, False), (True, 0, False), (False, 1, False), (False, 0, False), (True, 0, True), (False, 1, True)} <= rounds


@pytest.mark.parametrize("sizes,d", [((0, 4000, 0, 17, 1, 2500, 64), 392), ((1, 257, 5500, 0), 264), ((0, 0, 4000, 15, 241), 3208)])
@pytest.mark.parametrize("f,act", [(520, "swiglu"), (520, "relu"), (1160, "swiglu"), (1160, "relu")])
def test_uneven_slots(gpu_device, sizes, d, f, act):
    assert experts_take_tiles(sum(sizes), d, f, len(sizes), 1)[0]
    a = streamed.Layer(sum(sizes), d, f, len(sizes), 1, act, sizes=sizes)
    want, off = a.experts()
    a.gather()
    torch.cuda.synchronize()
    close(a.y[:-1], want, off)
    assert (a.y[-1] == 5.0).all()
    y = a.y.clone()
    a.combine()
    torch.cuda.synchronize()
    scale = a.weight.double().numpy()[:, :1]  # 1
    assert (scale == 1).all() and torch.equal(a.out[:-1], y[:-1][torch.from_numpy(a.inverse).cuda()])


@pytest.mark.parametrize("T,d,f", [(4000, 392, 1160), (2200, 3208, 1160), (5300, 392, 520), (4300, 3208, 520)])
@pytest.mark.parametrize("act", ("swiglu", "relu"))
def test_nan_and_infinity_stay_in_their_rows(gpu_device, T, d, f, act):
    assert experts_take_tiles(T, d, f, 2, 1)[0]
    a = streamed.Layer(T, d, f, 2, 1, act)
    a.combine()
    torch.cuda.synchronize()
    before = a.out[:-1].clone()
    bad = [3, T // 2, T - 1]
    a.dev["x"][3, 200] = float("nan")
    a.dev["x"][T // 2, 0] = float("inf")
    a.dev["x"][T - 1, d - 1] = -float("inf")
    a.combine()
    torch.cuda.synchronize()
    nan = torch.isnan(a.out[:-1])
    assert nan[bad].all() and int(nan.sum()) == len(bad) * d
    others = torch.ones(T, dtype=torch.bool)
    others[bad] = False
    assert torch.equal(a.out[:-1][others], before[others])


@pytest.mark.parametrize("T,d,f", [(3300, 264, 1032), (4300, 3208, 1032), (5300, 264, 520)])
@pytest.mark.parametrize("act", ("swiglu", "relu"))
def test_h_beyond_fp32_is_nan_and_large_h_is_not(gpu_device, T, d, f, act):
    """h passes fp32's range in one row, and only there is the result NaN."""
    assert experts_take_tiles(T, d, f, 1, 1)[0]
    a = streamed.Layer(T, d, f, 1, 1, act)
    x = np.zeros((T, d))
    x[:, 0] = 1.0
    top = 70 if act == "swiglu" else 120
    x[1, 0], x[2, 0] = 2.0 ** top, 2.0 ** (top - 20)
    w = np.zeros((f, d))
    w[:, 0] = np.linspace(0.5, 1.0, f) * (1 if act == "swiglu" else 2.0 ** 9)
    a.m1 = packed([w.astype(np.float32).astype(np.float64)])
    a.m3 = a.m1 if act == "swiglu" else None
    a.dev["x"] = as_device(x)
    a.combine()
    torch.cuda.synchronize()
    nan = torch.isnan(a.out[:-1])
    assert nan[1].all() and int(nan.sum()) == d and torch.isfinite(a.out[2]).all()


@pytest.mark.parametrize("T,d,f,S,k,act", [(2100, 264, 1160, 3, 2, "swiglu"), (2800, 3208, 520, 3, 2, "relu"), (4300, 3208, 520, 1, 1, "swiglu")])
def test_graph_replays_with_eager_work_between(gpu_device, T, d, f, S, k, act):
    assert experts_take_tiles(T, d, f, S, k)[0]
    a = streamed.Layer(T, d, f, S, k, act)
    x0, x1 = a.dev["x"].clone(), as_device(tokens(a.g, T, d))
    want = []
    for x in (x0, x1):
        a.dev["x"].copy_(x)
        a.combine()
        torch.cuda.synchronize()
        want.append(a.out.clone())
    assert not torch.equal(*want)
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


@pytest.mark.parametrize("T,d,f,S,k,act", [(3000, 392, 2056, 3, 2, "relu"), (2100, 3208, 2184, 2, 2, "swiglu"), (2800, 3208, 520, 3, 2, "swiglu")])
def test_the_same_bits_every_time(gpu_device, T, d, f, S, k, act):
    assert experts_take_tiles(T, d, f, S, k) == (True, True)
    a = streamed.Layer(T, d, f, S, k, act)
    a.gather()
    torch.cuda.synchronize()
    first = a.y.clone()
    other = torch.cuda.Stream()
    for i in range(6):
        a.ws.fill_(37 * i)
        a.y.fill_(5.0)
        torch.cuda.synchronize()
        a.gather(other if i % 2 else None)
        torch.cuda.synchronize()
        assert torch.equal(a.y, first)


@pytest.mark.parametrize("T,d,f,E,S,k,act", [(3000, 264, 520, 8, 4, 2, "swiglu"), (5000, 264, 1160, 16, 3, 1, "relu"), (3000, 3208, 520, 4, 2, 2, "relu")])
def test_layer_forward_in_one_call_and_in_four(gpu_device, T, d, f, E, S, k, act):
    assert experts_take_tiles(T, d, f, S, k)[0]
    streamed.test_layer_forward_in_one_call_and_in_four(gpu_device, T, d, f, E, S, k, act)
