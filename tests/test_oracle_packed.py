"""The oracle of matrices in 8 bits against torch's e4m3 and against itself."""
import numpy as np
import pytest
import torch

from oracle import packed as ref


def test_codes_and_values_are_those_of_e4m3():
    every = torch.arange(256, dtype=torch.uint8)
    want = every.view(torch.float8_e4m3fn).double().numpy()
    keep = ~np.isnan(want)
    assert np.array_equal(ref.values_of(every.numpy())[keep], want[keep])
    g = np.random.default_rng(0)
    x = np.concatenate((g.standard_normal(4000) * np.exp(g.uniform(-9, 5, 4000)), ref._MIDDLES, -ref._MIDDLES, ref.CODE_VALUES)).astype(np.float32)
    x = np.clip(x, -448, 448)
    assert np.array_equal(ref.codes_of(x.astype(np.float64)), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("top,e", [(0.0, -126), (448.0, 0), (448.0000001, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.7500001, -7), (2.0 ** -149, -126),
                                   (3.4028234663852886e38, 119), (1.75 * 2.0 ** 127, 119)])
def test_scales(top, e):
    assert ref.scale_exponent(top) == e


@pytest.mark.parametrize("N,K", [(8, 8), (136, 264), (256, 128)])
def test_pack_and_unpack_are_the_nearest_numbers(N, K):
    g = np.random.default_rng(N)
    w = g.standard_normal((N, K))
    back = ref.unpack(ref.pack(w), N, K)
    for i in range(0, N, 128):
        for j in range(0, K, 128):
            b = w[i:i + 128, j:j + 128]
            s = 2.0 ** ref.scale_exponent(np.abs(b).max())
            assert np.all(np.abs(back[i:i + 128, j:j + 128] - b) <= np.maximum(np.abs(b) * 2.0 ** -4, 2.0 ** -10 * s))
    assert np.array_equal(ref.unpack(ref.pack(back), N, K), back)  # (the largest may have become one that a smaller power holds)


def test_rows_share_the_matrix_format():
    g = np.random.default_rng(1)
    x = g.standard_normal((3, 300))
    q = ref.quantise_rows(x)
    for r in range(3):
        assert np.array_equal(ref.unpack(ref.pack(x[r:r + 1]), 1, 300), q[r:r + 1])
