"""The bound of kv_segments on the CPU: exact results and rounded ones are within it, results without some tokens are not, however long the context."""
import numpy as np
import pytest

from kv_segments import expected, misses


@pytest.mark.parametrize("length,dim,lost,dtype", [
    (30001, 128, 3000, "bf16"), (30001, 64, 10000, "bf16"), (20000, 64, 3000, "bf16"), (16000, 128, 64, "bf16"), (30001, 128, 32, "bf16"),
    (9001, 64, 32, "f32"), (9001, 64, 16, "f32")])
def test_what_is_left_out_is_found(length, dim, lost, dtype):
    g = np.random.default_rng(length + lost)
    for strong in (0.0, 1.0):
        scores = g.standard_normal((2, length)) * strong
        sees = np.ones((2, length), bool)
        want, seen = expected(scores, sees, dim)
        qk = np.full(2, 10.0 * strong)
        rounded = want * (1.0 + g.uniform(-1, 1, want.shape) * (2.0 ** -9 if dtype == "bf16" else 2.0 ** -24))
        assert misses(want, want, qk, seen, dim, dtype) == 0.0 and misses(rounded, want, qk, seen, dim, dtype) < 1.0
        for at in (0, length // 2 // 32 * 32, length - lost):
            less = sees.copy()
            less[:, at:at + lost] = False
            got, _ = expected(scores, less, dim)
            assert misses(got, want, qk, seen, dim, dtype) > 1.0
            twice = scores.copy()
            twice[:, at:at + lost] += np.log(2.0)  # the same tokens counted twice
            got, _ = expected(twice, sees, dim)
            assert misses(got, want, qk, seen, dim, dtype) > 1.0
