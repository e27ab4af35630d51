"""Calls of matrices in 8 bits on a machine without a GPU: extents and refusals."""
import pytest

import paper_2503_06823_amd as P

p = 4096  # a non-NULL address that must never be dereferenced


def test_bytes():
    assert P.emoe_matrix_bytes(8, 8) == 16384 + 256
    assert P.emoe_matrix_bytes(14336, 4096) == 112 * 32 * 16384 + 112 * 32
    assert P.emoe_matrix_bytes(1032, 2056) == 9 * 17 * 16384 + 256


@pytest.mark.parametrize("N,K,code", [(0, 8, P.EMOE_ERR_SHAPE), (8, -8, P.EMOE_ERR_SHAPE), (12, 8, P.EMOE_ERR_UNSUPPORTED), (8, 20, P.EMOE_ERR_UNSUPPORTED),
                                      (1 << 16, 1 << 15, P.EMOE_ERR_SHAPE), (2147483640, 8, P.EMOE_ERR_SHAPE), (16777216, 8, P.EMOE_ERR_SHAPE)])
def test_extents_out_of_range_are_refused_by_every_call(N, K, code):
    assert P.emoe_matrix_bytes(N, K, check=False) == code
    assert P.emoe_matrix_pack(1, N, K, "bf16", p, 2 * p, max(K, 8), stream=0, check=False) == code
    assert P.emoe_matrix_unpack(1, N, K, "bf16", p, 2 * p, max(K, 8), stream=0, check=False) == code
    d = P.make_matmul_desc(4, N, K)
    assert P.emoe_matmul_workspace_bytes(d, check=False) == code
    assert P.emoe_matmul(d, p, None, 2 * p, 3 * p, 4 * p, 1 << 40, stream=0, check=False) == code


@pytest.mark.parametrize("call,order", [(P.emoe_matrix_pack, 1), (P.emoe_matrix_unpack, -1)])
def test_pack_and_unpack_refuse(call, order):
    def rc(count=1, N=136, K=264, dtype="bf16", w=p, m=2 * p, stride=264):
        a = (w, m)[::order]
        return call(count, N, K, dtype, *a, stride, stream=0, check=False)
    assert rc(count=0, w=None, m=None) == P.EMOE_OK
    assert rc(count=-1) == P.EMOE_ERR_SHAPE and rc(count=65536) == P.EMOE_ERR_UNSUPPORTED
    assert rc(dtype="f8") == P.EMOE_ERR_UNSUPPORTED and rc(dtype=7) == P.EMOE_ERR_UNSUPPORTED
    assert rc(stride=256) == P.EMOE_ERR_SHAPE and rc(stride=268) == P.EMOE_ERR_UNSUPPORTED
    assert rc(w=None) == P.EMOE_ERR_NULL and rc(m=None) == P.EMOE_ERR_NULL
    assert rc(w=p + 8) == P.EMOE_ERR_UNSUPPORTED and rc(m=p + 8) == P.EMOE_ERR_UNSUPPORTED
    assert rc(w=p, m=p) == P.EMOE_ERR_SHAPE


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), P.EMOE_ERR_SHAPE), (dict(groups=0), P.EMOE_ERR_SHAPE), (dict(groups=65), P.EMOE_ERR_UNSUPPORTED), (dict(dtype="f32"), P.EMOE_ERR_UNSUPPORTED),
    (dict(dtype="f8"), P.EMOE_ERR_UNSUPPORTED), (dict(x_stride=256), P.EMOE_ERR_SHAPE), (dict(x_stride=268), P.EMOE_ERR_UNSUPPORTED),
    (dict(out_stride=128), P.EMOE_ERR_SHAPE), (dict(out_stride=140), P.EMOE_ERR_UNSUPPORTED), (dict(rows=6000000, x_stride=264), P.EMOE_ERR_SHAPE)])
def test_bad_descriptors_are_refused(kw, code):
    base = dict(rows=5, N=136, K=264, groups=2)
    base.update(kw)
    d = P.make_matmul_desc(**base)
    assert P.emoe_matmul_workspace_bytes(d, check=False) == code
    assert P.emoe_matmul(d, p, p, 2 * p, 3 * p, 4 * p, 1 << 40, stream=0, check=False) == code


def test_matmul_refuses():
    def rc(rows=5, groups=2, x=p, at=5 * p, m=2 * p, out=3 * p, ws=4 * p, less=0):
        d = P.make_matmul_desc(rows, 136, 264, groups)
        return P.emoe_matmul(d, x, at, m, out, ws, P.emoe_matmul_workspace_bytes(d) - less, stream=0, check=False)
    assert rc(rows=0, x=None, at=None, m=None, out=None, ws=None) == P.EMOE_OK
    assert rc(x=None) == P.EMOE_ERR_NULL and rc(m=None) == P.EMOE_ERR_NULL and rc(out=None) == P.EMOE_ERR_NULL
    assert rc(at=None) == P.EMOE_ERR_NULL
    assert rc(ws=None) == P.EMOE_ERR_WORKSPACE and rc(less=1) == P.EMOE_ERR_WORKSPACE
    for name in ("x", "m", "out", "ws"):
        assert rc(**{name: 7 * p + 8}) == P.EMOE_ERR_UNSUPPORTED
    assert rc(out=p) == P.EMOE_ERR_SHAPE and rc(out=2 * p) == P.EMOE_ERR_SHAPE and rc(ws=p) == P.EMOE_ERR_SHAPE
    assert rc(ws=2 * p) == P.EMOE_ERR_SHAPE and rc(ws=3 * p) == P.EMOE_ERR_SHAPE


def layer(**kw):
    base = dict(T=64, d_model=136, d_ff=264, E=8, k=2, S=4, dtype="f8", act="swiglu")
    base.update(kw)
    return P.make_desc(**base)


def test_layers_of_packed_experts():
    n = P.emoe_workspace_bytes(layer())
    assert n[1] >= 128 * (256 + 384) and n[1] % 256 == 0
    assert P.emoe_workspace_bytes(layer(T=0))[1] > 0
    # extents count in whole blocks
    assert P.emoe_workspace_bytes(layer(T=1 << 23, d_model=8, d_ff=8, k=1), check=False)[0] > 0
    assert P.emoe_workspace_bytes(layer(T=1 << 24, d_model=8, d_ff=8, k=1), check=False)[0] == P.EMOE_ERR_SHAPE
    assert P.emoe_workspace_bytes(layer(T=1 << 24, d_model=8, d_ff=8, k=1, dtype="bf16"), check=False)[0] > 0
    w = P.emoe_workspace_bytes(layer())[1]
    assert P.emoe_expert_ffn(layer(), p, p, p, None, p, p, p, w, stream=0, check=False) == P.EMOE_ERR_NULL
    assert P.emoe_expert_ffn(layer(act="relu"), p, p, p, p, p, p, p, w, stream=0, check=False) == P.EMOE_ERR_UNSUPPORTED
    assert P.emoe_expert_ffn(layer(), p, p, p, p, p, p, p, w - 1, stream=0, check=False) == P.EMOE_ERR_WORKSPACE


def test_cache_and_attention_take_no_packed_type():
    kv = P.make_kv_desc(10, 64, 8, 128, 4, 5)
    assert P.emoe_kv_append(kv, 4, "f8", p, p, p, p, stream=0, check=False) == P.EMOE_ERR_UNSUPPORTED
    assert P.emoe_kv_attention(kv, P.make_attention_desc(6, 32, 128, "f8", 2), p, p, p, p, p, p, p, 1 << 30, stream=0, check=False) == P.EMOE_ERR_UNSUPPORTED
