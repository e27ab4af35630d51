"""Calls of the paged 4-bit cache on a machine without a GPU: empty steps, and buffers that must not be the same."""
import pytest

import paper_2503_06823_amd as P

p = 4096  # a non-NULL address that must never be dereferenced


def kv(**kw):
    base = dict(pages=10, page_size=64, kv_heads=8, head_dim=128, rows=4, table_width=5)
    base.update(kw)
    return P.make_kv_desc(**base)


def attention(**kw):
    base = dict(T=6, q_heads=32, head_dim=128, dtype="bf16", max_new=2)
    base.update(kw)
    return P.make_attention_desc(**base)


@pytest.mark.parametrize("address", (None, p, p + 8))
def test_steps_without_tokens_or_requests_are_successes(address):
    """Whatever the buffers of nothing are: an empty tensor has no address."""
    a = address
    assert P.emoe_kv_append(kv(), 0, "bf16", a, a, a, p, stream=0) == P.EMOE_OK
    assert P.emoe_kv_read(kv(), 0, "bf16", p, a, a, a, stream=0) == P.EMOE_OK
    assert P.emoe_kv_attention(kv(), attention(T=0, max_new=0), a, a, a, a, a, a, a, 0, stream=0) == P.EMOE_OK
    assert P.emoe_kv_attention(kv(rows=0), attention(), a, a, a, a, a, a, a, 0, stream=0) == P.EMOE_OK


def test_bad_extents_are_refused_without_tokens_too():
    assert P.emoe_kv_append(kv(page_size=8), 0, "bf16", None, None, None, p, stream=0, check=False) == P.EMOE_ERR_UNSUPPORTED
    assert P.emoe_kv_append(kv(), 0, 7, None, None, None, p, stream=0, check=False) == P.EMOE_ERR_UNSUPPORTED
    assert P.emoe_kv_read(kv(head_dim=80), 0, "bf16", p, None, None, None, stream=0, check=False) == P.EMOE_ERR_UNSUPPORTED
    assert P.emoe_kv_attention(kv(), attention(T=0, max_new=1), p, p, p, p, p, p, p, 0, stream=0, check=False) == P.EMOE_ERR_SHAPE


PLAN = ("length", "new_len", "block_table", "free_pages", "counters", "cu_new", "slot", "position", "seq_len", "counters_out", "refused")
RELEASE = ("len_before", "length", "ended", "block_table", "free_pages", "counters", "counters_out")


def plan(**same):
    at = {n: p + 64 * i for i, n in enumerate(PLAN)}
    at.update({n: at[other] for n, other in same.items()})
    return P.emoe_kv_plan(kv(), 6, *[at[n] for n in PLAN], stream=0, check=False)


def release(**same):
    at = {n: p + 64 * i for i, n in enumerate(RELEASE)}
    at.update({n: at[other] for n, other in same.items()})
    return P.emoe_kv_release(kv(), at["len_before"], at["length"], at["ended"], 9, 1, at["block_table"], at["free_pages"], at["counters"],
                             at["counters_out"], stream=0, check=False)


@pytest.mark.parametrize("read", ("length", "new_len", "free_pages", "counters"))
@pytest.mark.parametrize("written", ("block_table", "cu_new", "slot", "position", "seq_len", "counters_out", "refused"))
def test_plan_reads_nothing_that_it_writes(read, written):
    """Workgroups read what another has written already or not: the lengths before and after a step have buffers of their own."""
    assert plan(**{written: read}) == P.EMOE_ERR_SHAPE


@pytest.mark.parametrize("read", ("len_before", "length", "ended", "block_table", "counters"))
@pytest.mark.parametrize("written", ("free_pages", "counters_out"))
def test_release_reads_nothing_that_it_writes(read, written):
    assert release(**{written: read}) == P.EMOE_ERR_SHAPE


def test_advance_refuses():
    q = p + 64
    assert P.emoe_kv_advance(kv(page_size=8), p, p, q, stream=0, check=False) == P.EMOE_ERR_UNSUPPORTED
    assert P.emoe_kv_advance(kv(), None, p, q, stream=0, check=False) == P.EMOE_ERR_NULL
    assert P.emoe_kv_advance(kv(), p, p, None, stream=0, check=False) == P.EMOE_ERR_NULL
    assert P.emoe_kv_advance(kv(), p, q, p, stream=0, check=False) == P.EMOE_ERR_SHAPE
    assert P.emoe_kv_advance(kv(), p, q, q, stream=0, check=False) == P.EMOE_ERR_SHAPE
    assert P.emoe_kv_advance(kv(rows=0), None, None, None, stream=0) == P.EMOE_OK
