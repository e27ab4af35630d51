"""emoe_matrix_pack and emoe_matrix_unpack: every byte of packed matrices against the oracle, and the numbers read back."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from oracle import packed as ref
from packed_util import as_device, bf16, weights

pytestmark = pytest.mark.gpu


def matrix(g, N, K, dtype):
    """Blocks over many magnitudes, with the values at which codes and powers turn."""
    w = g.standard_normal((N, K)) * np.exp(g.uniform(-20, 20, (-(-N // 128), -(-K // 128))).repeat(128, 0).repeat(128, 1)[:N, :K])
    w[0, :8] = [2.0 ** -10, -2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0, -17.0, 448.0, 0.0]  # ties of denormal and normal codes under 1
    w[1:8, :8] = 0.0
    if K > 128:
        w[:128, 128:256] = 0.0
        w[0, 128] = -0.0
    if N > 128:
        w[128:256, :128] *= 2.0 ** -8
        w[128, 0] = 448.0 * 2.0 ** 3  # the border of a power, and the number behind it
    if N > 128 and K > 128:
        w[128, 128] = np.abs(w[128:256, 128:256]).max() * 4
        w[128, 128] = 1.75 * 2.0 ** np.ceil(np.log2(w[128, 128])) * (1 + 2.0 ** -7)
    return bf16(w) if dtype == "bf16" else w.astype(np.float32).astype(np.float64)


def pack(matrices, dtype, gap=0):
    count, (N, K) = len(matrices), matrices[0].shape
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    wide = torch.full((count, N, K + gap), float("nan"), dtype=t, device="cuda")
    wide[:, :, :K] = torch.from_numpy(np.stack(matrices)).to("cuda", t)
    n = P.emoe_matrix_bytes(N, K)
    data = torch.full((count * n + 16,), 77, dtype=torch.uint8, device="cuda")
    P.emoe_matrix_pack(count, N, K, dtype, wide, data, K + gap)
    torch.cuda.synchronize()
    assert (data[count * n:] == 77).all()
    return data[:count * n].view(count, n)


def used(N, K):
    """Bytes of a packed matrix that mean something."""
    nb, kb = -(-N // 128), -(-K // 128)
    return nb * kb * 16384 + nb * (-(-kb // 4) * 4)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("count,N,K,gap", [(1, 8, 8, 0), (2, 128, 128, 8), (1, 136, 264, 0), (3, 200, 1032, 24), (1, 384, 520, 0), (5, 16, 640, 0)])
def test_pack_and_unpack(gpu_device, count, N, K, gap, dtype):
    g = np.random.default_rng(N + K)
    ws = [matrix(g, N, K, dtype) for _ in range(count)]
    data = pack(ws, dtype, gap)
    for got, w in zip(data.cpu().numpy(), ws):
        assert np.array_equal(got[:used(N, K)], ref.pack(w)[:used(N, K)])
    for out_type in ("bf16", "f32"):
        out = torch.full((count, N, K + gap), 5.0, dtype=torch.float32 if out_type == "f32" else torch.bfloat16, device="cuda")
        P.emoe_matrix_unpack(count, N, K, out_type, data, out, K + gap)
        torch.cuda.synchronize()
        for o, d in zip(out, data.cpu().numpy()):
            assert np.array_equal(o[:, :K].double().cpu().numpy(), ref.unpack(d, N, K))
        assert (out[:, :, K:] == 5.0).all()


def test_largest_and_smallest_numbers_stay_finite(gpu_device):
    top = float(torch.finfo(torch.float32).max)
    w = np.zeros((128, 640))
    w[3, 0], w[4, 1] = top, -top           # 448 * 2^119
    w[:, 128] = 1.75 * 2.0 ** 127          # the largest that its code holds
    w[5, 256:384] = 2.0 ** -149            # denormal numbers
    w[6, 384], w[6, 385] = 448 * 2.0 ** -126, 2.0 ** -135
    w[0, 512] = 2.0 ** -126
    got = pack([w], "f32").cpu().numpy()[0]
    assert np.array_equal(got[:used(128, 640)], ref.pack(w)[:used(128, 640)])
    out = torch.empty((128, 640), dtype=torch.float32, device="cuda")
    P.emoe_matrix_unpack(1, 128, 640, "f32", torch.from_numpy(got).cuda(), out)
    back = out.double().cpu().numpy()
    assert np.isfinite(back).all() and back[3, 0] == 1.75 * 2.0 ** 127 and back[4, 1] == -1.75 * 2.0 ** 127
    assert np.array_equal(back, ref.unpack(got, 128, 640))


@pytest.mark.parametrize("value", (np.nan, np.inf, -np.inf))
def test_a_block_with_an_infinity_or_nan_is_nan_and_no_other_is(gpu_device, value):
    g = np.random.default_rng(3)
    w = bf16(g.standard_normal((256, 256)))
    w[200, 17] = value
    data = pack([w], "bf16")
    out = torch.empty((256, 256), dtype=torch.bfloat16, device="cuda")
    P.emoe_matrix_unpack(1, 256, 256, "bf16", data, out)
    nan = torch.isnan(out).cpu().numpy()
    assert nan[128:, :128].all() and nan.sum() == 128 * 128


def test_bytes(gpu_device):
    for N, K in ((8, 8), (128, 128), (136, 520), (14336, 4096), (1032, 2808)):
        assert P.emoe_matrix_bytes(N, K) == ref.matrix_bytes(N, K)


@pytest.mark.parametrize("N,K,count", [(136, 264, 2), (8, 8, 3), (128, 128 * 64, 1), (264, 8208, 2)])
def test_every_byte_of_a_matrix_is_written(gpu_device, N, K, count):
    """Whatever the room held: the bytes depend on the input only."""
    w = np.stack([weights(np.random.default_rng(N + i), N, K) for i in range(count)])
    room = torch.full((count * P.emoe_matrix_bytes(N, K) + 256,), 171, dtype=torch.uint8, device="cuda")
    P.emoe_matrix_pack(count, N, K, "bf16", as_device(w), room)
    got = room.cpu().numpy()
    assert np.array_equal(got[:-256], np.concatenate([ref.pack(m) for m in w])) and (got[-256:] == 171).all()
