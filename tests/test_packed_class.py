"""PackedMatrices on a machine without a GPU: what it refuses before anything is enqueued, and what it hands to the library."""
import pytest
import torch

import paper_2503_06823_amd as P
from paper_2503_06823_amd import binding as B

N, K = 136, 264
BF16 = dict(dtype=torch.bfloat16)
I32 = dict(dtype=torch.int32)


@pytest.fixture
def calls(monkeypatch):
    """The library's calls that enqueue work, which are noted and not made."""
    noted = []
    for name in ("emoe_matrix_pack", "emoe_matrix_unpack", "emoe_matmul"):
        monkeypatch.setattr(B, name, lambda *a, name=name, **kw: noted.append((name, a)))
    return noted


def made(count=1):
    return P.PackedMatrices.allocate(count, N, K, device="cpu")


def test_pack_hands_over_type_and_stride(calls):
    for w, count, dtype, stride in [
        (torch.zeros((N, K), **BF16), 1, P.EMOE_BF16, K), (torch.zeros((3, N, K)), 3, P.EMOE_F32, K),
        (torch.zeros((2, N, K + 16), **BF16)[:, :, 8:K + 8], 2, P.EMOE_BF16, K + 16), (torch.zeros((N + 8, K), **BF16)[8:], 1, P.EMOE_BF16, K),
        (torch.zeros((1, N, K), **BF16), 1, P.EMOE_BF16, K)]:
        calls.clear()
        m = P.PackedMatrices.pack(w)
        (name, a), = calls
        assert name == "emoe_matrix_pack" and a[:4] == (count, N, K, dtype) and a[4] is w and a[5] is m.data and a[6] == stride
        assert m.count == count and m.data.shape == (count, P.emoe_matrix_bytes(N, K)) and m.data.dtype is torch.uint8


BAD_MATRICES = [
    torch.zeros((2, N, K)), torch.zeros((N, K), dtype=torch.float16), torch.zeros((N, K), dtype=torch.float64), torch.zeros((K, N)),
    torch.zeros((K, N)).t(), torch.zeros((N, 2 * K))[:, ::2], torch.zeros((1, K)).expand(N, K), torch.zeros((N, K), device="meta"),
    torch.zeros(N * K), torch.zeros((1, 1, N, K)), None, [[1.0]]]


@pytest.mark.parametrize("bad", BAD_MATRICES)
def test_write_and_read_refuse(calls, bad):
    for call in (made().write, made().read):
        with pytest.raises(ValueError):
            call(bad)
    assert not calls


def test_matrices_at_another_distance_than_their_rows_are_refused(calls):
    with pytest.raises(ValueError):
        made(2).write(torch.zeros((2, N + 1, K))[:, :N])
    with pytest.raises(ValueError):
        made(2).write(torch.zeros((N, 2, K)).transpose(0, 1))
    assert not calls


@pytest.mark.parametrize("w", [torch.zeros(8), None, "w", torch.zeros((1, 1, 8, 8))])
def test_pack_refuses(calls, w):
    with pytest.raises(ValueError):
        P.PackedMatrices.pack(w)


@pytest.mark.parametrize("shape", [(7, 8), (8, 12), (0, 8)])
def test_extents_that_the_library_does_not_take(calls, shape):
    with pytest.raises(P.EmoeError):
        P.PackedMatrices.pack(torch.zeros(shape))


def test_data_of_another_size_is_refused():
    n = P.emoe_matrix_bytes(N, K)
    for data in (torch.zeros((1, n - 1), dtype=torch.uint8), torch.zeros((1, n), dtype=torch.int8), torch.zeros(n, dtype=torch.uint8),
                 torch.zeros((0, n), dtype=torch.uint8), torch.zeros((1, 2 * n), dtype=torch.uint8)[:, ::2], None):
        with pytest.raises(ValueError):
            P.PackedMatrices(N, K, data)


def rows(n, width):
    return torch.zeros((n, width), **BF16)


def test_matmul_hands_over_rows_and_strides(calls):
    for count, x, out, at, want in [
        (1, rows(5, K), rows(5, N), None, (5, K, N)), (1, rows(5, K + 8)[:, :K], rows(5, N + 24)[:, 24:], None, (5, K + 8, N + 24)),
        (1, rows(1, K + 3)[:, :K], rows(1, N), None, (1, K, N)), (3, rows(5, K), rows(5, N), torch.zeros(4, **I32), (5, K, N)),
        (1, rows(10, K)[::2], rows(5, N), torch.zeros(2, **I32), (5, 2 * K, N)), (1, rows(0, K), rows(0, N), None, (0, K, N))]:
        calls.clear()
        m = made(count)
        ws = m.workspace(5)
        assert m.matmul(x, out, ws, at) is out
        (name, (desc, *a)), = calls
        assert (desc.rows, desc.x_stride, desc.out_stride) == want
        assert (desc.N, desc.K, desc.groups, desc.dtype, desc.reserved) == (N, K, count, P.EMOE_BF16, 0)
        assert a[0] is x and a[1] is at and a[2] is m.data and a[3] is out and a[4] is ws and a[5] == ws.numel()


def test_matmul_refuses(calls):
    m, three = made(), made(3)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    x, out, at = rows(5, K), rows(5, N), torch.zeros(4, **I32)
    bad_x = [rows(5, K - 8), x.float(), x.half(), x[0], x[None], rows(K, 5).t(), rows(5, 2 * K)[:, ::2], rows(1, K).expand(5, K), x.to("meta"), None]
    bad_out = [rows(5, N + 8), rows(4, N), rows(6, N), out.float(), rows(N, 5).t(), rows(1, N).expand(5, N), out.to("meta"), None]
    bad_ws = [ws.int(), ws[::2], ws.to("meta"), None]
    bad_at = [None, at[:3], torch.zeros(5, **I32), at.long(), torch.zeros(8, **I32)[::2], at[None], at.to("meta"), [0, 1, 2, 3]]
    for call in ([lambda b=b: m.matmul(b, out, ws) for b in bad_x] + [lambda b=b: m.matmul(x, b, ws) for b in bad_out]
                 + [lambda b=b: m.matmul(x, out, b) for b in bad_ws] + [lambda b=b: three.matmul(x, out, ws, b) for b in bad_at]
                 + [lambda: m.matmul(x, out, ws, at)]):
        with pytest.raises(ValueError):
            call()
    assert not calls


def test_another_current_device_is_refused(calls, monkeypatch):
    m = made()
    m._device = torch.device("cuda", 1)  # the tensors' devices are compared with it first, so this asks the check itself
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        m._check_device()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    m._check_device()


def test_workspace_covers_fewer_rows():
    for count in (1, 3, 64):
        m = made(count)
        sizes = [m.workspace_bytes(n) for n in (0, 1, 16, 17, 36 * count, 37 * count, 128 * count, 129 * count, 1000 * count)]
        assert sizes == sorted(sizes)
        assert m.workspace(16).numel() >= sizes[2]
