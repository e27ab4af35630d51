"""KvCache on a machine without a GPU: what it refuses before anything is enqueued, and what it hands to the library."""
import pytest
import torch

import paper_2503_06823_amd as P
from paper_2503_06823_amd import binding as B

I32 = dict(dtype=torch.int32)
HEADS, DIM = 2, 64


@pytest.fixture
def made(monkeypatch):
    """A cache of three requests and two layers in host memory, and the library's calls, which are noted and not made."""
    calls = []
    for name in ("emoe_kv_plan", "emoe_kv_append", "emoe_kv_attention", "emoe_kv_release", "emoe_kv_advance"):
        if hasattr(B, name):
            monkeypatch.setattr(B, name, lambda *a, name=name, **kw: calls.append((name, a)))
    kv = P.KvCache.allocate(2, 3, 100, 20, 16, HEADS, DIM, 10, device="cpu")
    return kv, calls


def rows(T, heads=HEADS, dim=DIM, dtype=torch.bfloat16):
    return torch.zeros((T, heads, dim), dtype=dtype)


def planned(kv, T=6):
    kv.plan(torch.tensor([T, 0, 0], **I32), T)
    return kv


@pytest.mark.parametrize("new_len,T", [
    (torch.zeros(3, dtype=torch.int64), 6), (torch.zeros(3, dtype=torch.bool), 6), (torch.zeros(2, **I32), 6), (torch.zeros(4, **I32), 6),
    (torch.zeros((3, 1), **I32), 6), (torch.zeros(6, **I32)[::2], 6), ([1, 2, 3], 6), (None, 6), (torch.zeros(3, **I32), -1),
    (torch.zeros(3, **I32), 11), (torch.zeros(3, device="meta", **I32), 6)])
def test_plan_refuses(made, new_len, T):
    kv, calls = made
    with pytest.raises(ValueError):
        kv.plan(new_len, T)
    assert not calls and kv.T == 0


BAD_ROWS = [
    rows(5),                                              # fewer than the step has
    rows(6, heads=1), rows(6, heads=3), rows(6, dim=128), rows(6).reshape(6, -1),
    rows(6, dtype=torch.float32), rows(6, dtype=torch.float16),
    torch.zeros((6, DIM, HEADS), dtype=torch.bfloat16).transpose(1, 2),       # elements apart
    torch.zeros((6, 2 * HEADS, DIM), dtype=torch.bfloat16)[:, ::2],           # heads apart
    torch.zeros((HEADS, 6, DIM), dtype=torch.bfloat16).transpose(0, 1),       # heads further apart than tokens
    torch.zeros((1, HEADS, DIM), dtype=torch.bfloat16).expand(6, -1, -1),     # one row for all
    rows(6).to("meta"), None,
]


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_append_refuses(made, bad):
    kv, calls = made
    planned(kv)
    calls.clear()
    for k, v in ((bad, rows(6)), (rows(6), bad)):
        with pytest.raises(ValueError):
            kv.append(0, k, v)
    assert not calls


@pytest.mark.parametrize("bad", [b for b in BAD_ROWS if b is None or b.dim() != 3 or b.shape[1] != 1])
def test_attend_refuses(made, bad):
    kv, calls = made
    planned(kv)
    calls.clear()
    for q, out in ((bad, rows(6)), (rows(6), bad)):
        with pytest.raises(ValueError):
            kv.attend(0, q, out, 6)
    for q, out in ((rows(6, heads=4), rows(6, heads=2)), (rows(6, heads=3), rows(6, heads=3)), (rows(6, heads=0), rows(6, heads=0))):
        with pytest.raises(ValueError):
            kv.attend(0, q, out, 6)
    assert not calls


@pytest.mark.parametrize("ended", [torch.zeros(3, dtype=torch.bool), torch.zeros(3, dtype=torch.int64), torch.zeros(2, **I32), torch.zeros((3, 1), **I32),
                                   torch.zeros(6, **I32)[::2], [0, 0, 1], torch.zeros(3, device="meta", **I32)])
def test_release_refuses(made, ended):
    kv, calls = made
    planned(kv)
    calls.clear()
    with pytest.raises(ValueError):
        kv.release(ended)
    assert not calls


def test_what_is_taken(made):
    """Slices of a wider row, buffers of more rows than the step has, a step of one row or none."""
    kv, calls = made
    planned(kv)
    wide = torch.zeros((8, 4 + 2 * HEADS, DIM), dtype=torch.bfloat16)
    kv.append(1, wide[:, 4:4 + HEADS], wide[:, 4 + HEADS:])
    name, a = calls[-1]
    assert name == "emoe_kv_append" and a[1] == 6 and a[7] == a[8] == wide.stride(0)
    out = rows(6, heads=4)
    assert kv.attend(1, wide[:, :4], out, 9) is out
    at = calls[-1][1][1]
    assert (at.T, at.max_new, at.q_stride, at.out_stride) == (6, 6, wide.stride(0), 4 * DIM)  # no request has more than the step
    planned(kv, 1)
    one = torch.zeros((1, HEADS, DIM), dtype=torch.bfloat16).as_strided((1, HEADS, DIM), (8, DIM, 1))  # a row's own stride says nothing
    kv.append(0, one, one)
    assert calls[-1][1][7] == HEADS * DIM
    planned(kv, 0)
    empty = rows(0)
    kv.append(0, empty, empty)
    assert calls[-1][1][1] == 0
    kv.attend(0, empty, empty, 1)
    assert calls[-1][1][1].T == 0 and calls[-1][1][1].max_new == 0
    kv.release(torch.zeros(3, **I32))
    kv.release()


def test_fp32_rows(made):
    kv = P.KvCache.allocate(1, 3, 100, 20, 16, HEADS, DIM, 10, dtype="f32", device="cpu")
    planned(kv)
    kv.append(0, rows(6, dtype=torch.float32), rows(6, dtype=torch.float32))
    with pytest.raises(ValueError):
        kv.append(0, rows(6), rows(6))


def test_a_step_leaves_every_buffer_in_its_place(made):
    """The next step reads and writes where this one did, so that a captured step replays as the next."""
    kv, calls = made

    def step():
        calls.clear()
        planned(kv)
        kv.release(torch.zeros(3, **I32))
        keep = [id(t) for t in (*kv.length, *kv.counters)]
        return [name for name, _ in calls], keep, [[id(x) for x in a if isinstance(x, torch.Tensor) and x.numel() != 3 or x is kv.length[0]] for _, a in calls]

    first = step()
    assert first[0] == ["emoe_kv_plan", "emoe_kv_release", "emoe_kv_advance"]  # nothing of it is torch's
    assert step() == first
