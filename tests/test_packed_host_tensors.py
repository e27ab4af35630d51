"""Calls of matrices in 8 bits with tensors of the host's memory, whose addresses no kernel may get: refused before the library is called."""
import numpy as np
import pytest
import torch

import paper_2503_06823_amd as P
from paper_2503_06823_amd import binding as B

N, K = 136, 264
p = 4096  # an address that says nothing about where it lies
BF16 = dict(dtype=torch.bfloat16)


class Library:
    """The extents' calls are the library's; whatever would enqueue work is noted and not made."""
    def __init__(self, real):
        self.real, self.made = real, []

    def __getattr__(self, name):
        if name in ("emoe_matrix_pack", "emoe_matrix_unpack", "emoe_matmul"):
            return lambda *a: self.made.append((name, a)) or P.EMOE_OK
        return getattr(self.real, name)


@pytest.fixture
def library(monkeypatch):
    it = Library(B.lib())
    monkeypatch.setattr(B, "lib", lambda: it)
    monkeypatch.setattr(B, "_stream_addr", lambda stream: 0)
    return it


@pytest.mark.parametrize("w", [torch.zeros((N, K), **BF16), torch.zeros((3, N, K)), torch.nn.Parameter(torch.zeros((N, K)))])
def test_a_checkpoint_in_host_memory_is_not_packed(library, w):
    with pytest.raises(ValueError, match="GPU"):
        P.PackedMatrices.pack(w)
    assert not library.made


def test_the_class_refuses_host_tensors(library):
    m = P.PackedMatrices.allocate(1, N, K, device="cpu")
    x, out, ws = torch.zeros((5, K), **BF16), torch.zeros((5, N), **BF16), m.workspace(5)
    for call in (lambda: m.write(torch.zeros((N, K))), lambda: m.read(torch.zeros((N, K))), lambda: m.matmul(x, out, ws),
                 lambda: m.matmul(x, out, ws, torch.tensor([0, 5], dtype=torch.int32)), lambda: m.matmul(x[:0], out[:0], ws)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    assert not library.made


HOST = [torch.zeros(1 << 16, dtype=torch.uint8), np.zeros(1 << 16, dtype=np.uint8), torch.zeros(1 << 16, dtype=torch.uint8, device="meta")]


@pytest.mark.parametrize("bad", HOST, ids=("tensor", "array", "meta"))
def test_every_buffer_of_the_calls_is_looked_at(library, bad):
    desc = P.make_matmul_desc(5, N, K)
    for i in range(5):
        buffers = [i_ * p for i_ in range(1, 6)]
        buffers[i] = bad
        with pytest.raises(ValueError, match="GPU"):
            P.emoe_matmul(desc, *buffers, 1 << 20, stream=0)
    for call in (P.emoe_matrix_pack, P.emoe_matrix_unpack):
        for a in ((bad, p), (p, bad)):
            with pytest.raises(ValueError, match="GPU"):
                call(1, N, K, "bf16", *a, stream=0)
    assert not library.made


def test_addresses_and_none_are_handed_over(library):
    P.emoe_matmul(P.make_matmul_desc(5, N, K), p, None, 2 * p, 3 * p, 4 * p, 1 << 20, stream=0)
    P.emoe_matrix_pack(1, N, K, "bf16", p, 2 * p, stream=0)
    (_, a), (_, b) = library.made
    assert a[1:6] == (p, None, 2 * p, 3 * p, 4 * p) and b[4:7] == (p, K, 2 * p)
