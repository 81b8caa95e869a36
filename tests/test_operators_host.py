"""Packed attention, its gradient and the paged cache on the host: refusals of
the C entry points and of the binding (fake pointers are never dereferenced),
and the plain forms the GPU tests compare with."""

import ctypes
import math

import pytest
import torch

import attn_ref as ref


@pytest.fixture(scope="module")
def P():
    import paper_2609_32814_amd as P
    import paper_2609_32814_amd.binding  # noqa: F401
    return P


@pytest.fixture(scope="module")
def E(P):
    return {v: k for k, v in P.binding.STATUS_NAMES.items()}


V = ctypes.c_void_p


def shape(P, **kw):
    base = dict(batch=2, seq_len=100, n_heads=4, n_kv_heads=2, head_dim=64, q=4, law=0)
    base.update(kw)
    return P.binding._CAttnShape(**base)


def fwd(P, sh, dt=1, ot=1, ptr=16, pack=16, lse=None, nbytes=1 << 30):
    p = V(ptr) if ptr else None
    return P.binding.LIB.star_attn_packed_fwd(ctypes.byref(sh), V(pack) if pack else None, nbytes, p, p, p, dt, p, ot,
                                              V(lse) if lse else None, 0, None)


def bwd(P, sh, dt=1, ot=1, gt=1, ptr=16, lse=16, ws=16, nbytes=1 << 30, ws_bytes=1 << 30):
    p = V(ptr) if ptr else None
    return P.binding.LIB.star_attn_packed_bwd(ctypes.byref(sh), V(16), nbytes, p, p, p, p, dt, p, ot, V(lse) if lse else None,
                                              p, p, p, gt, 0, V(ws) if ws else None, ws_bytes, None)


def pages(P, **kw):
    base = dict(n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, batch=2, max_pages=4, type=1, K=16, V=16, K_scale=16,
                V_scale=16, page_table=16)
    base.update(kw)
    return P.binding._CKvPages(**base)


def append(P, pg, T=5, ptr=16, cu=16, dt=1):
    p = V(ptr) if ptr else None
    return P.binding.LIB.star_kv_append(ctypes.byref(pg), V(cu) if cu else None, V(16), T, p, p, dt, None)


def read(P, pg, T=5, ptr=16, dt=1):
    p = V(ptr) if ptr else None
    return P.binding.LIB.star_kv_read(ctypes.byref(pg), V(16), V(16), T, p, p, dt, 0, None)


def decode(P, sh, pg, ptr=16, types=16, dt=1, ot=1, ws=16, ws_bytes=1 << 30):
    p = V(ptr) if ptr else None
    return P.binding.LIB.star_attn_decode_paged(ctypes.byref(sh), ctypes.byref(pg), V(types) if types else None, V(16), p, dt,
                                                p, ot, V(ws) if ws else None, ws_bytes, None)


def test_packed_refusals(P, E):
    for call in (fwd, bwd):
        assert call(P, shape(P, law=3)) == E["STAR_ERR_UNSUPPORTED"]
        assert call(P, shape(P, law=9)) == E["STAR_ERR_ARG"]
        assert call(P, shape(P, head_dim=96, q=2)) == E["STAR_ERR_UNSUPPORTED"]
        assert call(P, shape(P, q=16)) == E["STAR_ERR_UNSUPPORTED"]       # groups of 4
        assert call(P, shape(P, n_kv_heads=3)) == E["STAR_ERR_SHAPE"]
        assert call(P, shape(P, seq_len=(1 << 18) + 1)) == E["STAR_ERR_SHAPE"]
        assert call(P, shape(P, batch=(1 << 14) + 1)) == E["STAR_ERR_SHAPE"]
        assert call(P, shape(P, batch=-1)) == E["STAR_ERR_SHAPE"]
        assert call(P, shape(P, seq_len=2, n_heads=1 << 21, n_kv_heads=1 << 21)) == E["STAR_ERR_SHAPE"]  # a row of Q
        assert call(P, shape(P), dt=0) == E["STAR_ERR_DTYPE"]
        assert call(P, shape(P), ot=7) == E["STAR_ERR_DTYPE"]
        assert call(P, shape(P), ptr=None) == E["STAR_ERR_ARG"]
        assert call(P, shape(P), ptr=24) == E["STAR_ERR_ALIGN"]
        assert call(P, shape(P), lse=18) == E["STAR_ERR_ALIGN"]
        assert call(P, shape(P), nbytes=P.star_attn_pack_bytes(4, 100, 2) - 1) == E["STAR_ERR_WORKSPACE"]
        assert call(P, shape(P, seq_len=0), ptr=None) == 0
    assert fwd(P, shape(P), pack=None) == E["STAR_ERR_WORKSPACE"]
    assert fwd(P, shape(P), pack=24) == E["STAR_ERR_ALIGN"]
    assert bwd(P, shape(P), gt=3) == E["STAR_ERR_DTYPE"]
    assert bwd(P, shape(P), lse=None) == E["STAR_ERR_ARG"]
    assert bwd(P, shape(P), ws=None) == E["STAR_ERR_WORKSPACE"]
    need = P.star_attn_packed_bwd_workspace_bytes(P.AttnShape(2, 100, 4, 2, 64, 4))
    assert need >= 4 * 4 * 100
    assert bwd(P, shape(P), ws_bytes=need - 1) == E["STAR_ERR_WORKSPACE"]
    assert P.star_attn_packed_bwd_workspace_bytes(P.AttnShape(2, 100, 4, 2, 64, 4, "graph")) == 0


def test_pack_refusals(P, E):
    lib = P.binding.LIB
    need = P.star_attn_pack_bytes(4, 100, 2)
    assert need > 0 and P.star_attn_pack_bytes(17, 100, 2) == 0 and P.star_attn_pack_bytes(4, -1, 2) == 0
    call = lambda q=4, T=100, n=2, t=16, cu=16, pack=16, nb=need: lib.star_attn_pack(
        q, T, n, V(t) if t else None, V(cu) if cu else None, V(pack) if pack else None, nb, None)
    assert call(q=0) == E["STAR_ERR_ARG"] and call(q=17) == E["STAR_ERR_ARG"]
    assert call(T=(1 << 18) + 1) == E["STAR_ERR_SHAPE"] and call(n=-1) == E["STAR_ERR_SHAPE"]
    assert call(t=None) == E["STAR_ERR_ARG"] and call(cu=None) == E["STAR_ERR_ARG"]
    assert call(pack=None) == E["STAR_ERR_WORKSPACE"] and call(nb=need - 1) == E["STAR_ERR_WORKSPACE"]
    assert call(t=18) == E["STAR_ERR_ALIGN"] and call(pack=8) == E["STAR_ERR_ALIGN"]


def test_cache_refusals(P, E):
    sh = shape(P, seq_len=64)
    for call in (append, read, lambda P, pg, **kw: decode(P, sh, pg, **kw)):
        assert call(P, pages(P, type=4)) == E["STAR_ERR_ARG"]
        assert call(P, pages(P, head_dim=80)) == E["STAR_ERR_UNSUPPORTED"]
        for size in (0, 4, 24, 2048):
            assert call(P, pages(P, page_size=size)) == E["STAR_ERR_UNSUPPORTED"]
        assert call(P, pages(P, n_pages=-1)) == E["STAR_ERR_SHAPE"]
        assert call(P, pages(P, max_pages=1 << 27)) == E["STAR_ERR_SHAPE"]
        assert call(P, pages(P, K=None)) == E["STAR_ERR_ARG"]
        assert call(P, pages(P, K_scale=None)) == E["STAR_ERR_ARG"]
        assert call(P, pages(P, page_table=None)) == E["STAR_ERR_ARG"]
        assert call(P, pages(P, V=24)) == E["STAR_ERR_ALIGN"]
        assert call(P, pages(P, V_scale=24)) == E["STAR_ERR_ALIGN"]
        assert call(P, pages(P), ptr=None) == E["STAR_ERR_ARG"]
        assert call(P, pages(P), ptr=24) == E["STAR_ERR_ALIGN"]
        assert call(P, pages(P), dt=0) == E["STAR_ERR_DTYPE"]
    for call in (append, read):
        assert call(P, pages(P), T=-1) == E["STAR_ERR_SHAPE"]
        assert call(P, pages(P), T=0, ptr=None) == 0
    assert append(P, pages(P), cu=None) == E["STAR_ERR_ARG"]
    assert decode(P, shape(P, seq_len=65), pages(P)) == E["STAR_ERR_SHAPE"]
    assert decode(P, shape(P, seq_len=64, batch=3), pages(P)) == E["STAR_ERR_SHAPE"]
    assert decode(P, shape(P, seq_len=64, head_dim=128), pages(P)) == E["STAR_ERR_SHAPE"]
    assert decode(P, shape(P, seq_len=0), pages(P, max_pages=0)) == E["STAR_ERR_SHAPE"]
    assert decode(P, shape(P, seq_len=64, law=3), pages(P)) == E["STAR_ERR_UNSUPPORTED"]
    assert decode(P, sh, pages(P), types=None) == E["STAR_ERR_ARG"]
    assert decode(P, sh, pages(P), types=20) == E["STAR_ERR_ALIGN"]
    assert decode(P, sh, pages(P), ot=5) == E["STAR_ERR_DTYPE"]
    assert decode(P, sh, pages(P), ws=None) == E["STAR_ERR_WORKSPACE"]
    need = P.star_attn_decode_paged_workspace_bytes(P.AttnShape(2, 64, 4, 2, 64, 4))
    assert need > 0 and decode(P, sh, pages(P), ws_bytes=need - 1) == E["STAR_ERR_WORKSPACE"]
    assert decode(P, shape(P, seq_len=64, batch=0), pages(P, batch=0), ptr=None) == 0


def test_binding_refuses_bad_tensors(P):
    b16, i32 = torch.bfloat16, torch.int32
    sh = P.AttnShape(1, 8, 2, 1, 64, 2)
    Q, K = torch.zeros((8, 2, 64), dtype=b16), torch.zeros((8, 1, 64), dtype=b16)
    pack, lse = torch.zeros(4096, dtype=torch.uint8), torch.zeros((2, 8))
    cu, t = torch.zeros(2, dtype=i32), torch.zeros(8, dtype=i32)
    with pytest.raises(TypeError):
        P.star_attn_pack(2, t, cu.long())
    with pytest.raises(ValueError):
        P.star_attn_pack(2, t, cu[:0])
    with pytest.raises(ValueError):
        P.star_attn_pack(2, t, cu)                                          # CPU tensors
    with pytest.raises(ValueError):
        P.star_attn_packed_fwd(sh, pack, Q, K[:4], K)
    with pytest.raises(TypeError):
        P.star_attn_packed_fwd(sh, pack, Q.float(), K, K)
    with pytest.raises(ValueError):
        P.star_attn_packed_fwd(sh, pack, Q.transpose(0, 1).contiguous().transpose(0, 1), K, K)  # strides
    with pytest.raises(ValueError):
        P.star_attn_packed_fwd(sh, pack, Q, K, K)                           # CPU tensors
    with pytest.raises(ValueError):
        P.star_attn_packed_bwd(sh, pack, Q, Q, K, K, Q, lse, dQ=Q)          # one gradient alone
    with pytest.raises(TypeError):
        P.star_attn_packed_bwd(sh, pack, Q, Q, K, K, Q, lse.double())
    pg = torch.zeros((4, 1, 8, 64), dtype=b16)
    table, sc = torch.zeros((1, 2), dtype=i32), torch.zeros((4, 1, 8), dtype=torch.uint8)
    with pytest.raises(ValueError):
        P.KVPages(pg, pg, table, sc, sc)                                    # scales of bf16 pages
    with pytest.raises(ValueError):
        P.KVPages(pg.to(torch.int8), pg.to(torch.int8), table)              # none of int8 pages
    with pytest.raises(TypeError):
        P.KVPages(pg.float(), pg.float(), table)
    with pytest.raises(TypeError):
        P.KVPages(pg, pg, table.long())
    with pytest.raises(ValueError):
        P.KVPages(pg, pg[:2], table)
    kv = P.KVPages(pg, pg, table)
    assert kv.capacity == 16 and "bfloat16" in repr(kv)
    with pytest.raises(ValueError):
        P.star_kv_append(kv, cu, cu[:1], K, K)                              # CPU tensors
    with pytest.raises(ValueError):
        P.star_kv_read(kv, cu, cu[:1], 3, K=K)                              # one of two
    with pytest.raises(ValueError):
        P.star_attn_decode_paged(P.AttnShape(1, 16, 2, 1, 64, 2), kv, t, cu[:1], Q[:1])


@pytest.mark.parametrize("law,q,H,Hkv", [("star", 4, 2, 1), ("dense", 1, 2, 2), ("tensor2", 4, 4, 2)])
def test_reference_gradient_against_differences(law, q, H, Hkv):
    """The formula the GPU's gradient is held to is the derivative of the
    forward: central differences along random directions, in 64 bits (error
    h^2 of a function whose derivatives are of order one)."""
    g = torch.Generator().manual_seed(q)
    D, cu = 8 * q if q > 1 else 16, [0, 1, 12, 12, 20]
    T = 22
    r = lambda h: torch.randn((T, h, D), generator=g, dtype=torch.float64)
    Q, K, V, dO = r(H), r(Hkv), r(Hkv), r(H)
    types = torch.randint(0, q, (T,), generator=g).to(torch.int32)
    types[5] = -1
    O, lse, _ = ref.forward(law, q, types, cu, Q, K, V)
    grads, _ = ref.backward(law, q, types, cu, dO, Q, K, V, O, lse)
    h = 1e-5
    for n, x in enumerate((Q, K, V)):
        d = torch.randn(x.shape, generator=g, dtype=torch.float64)
        side = []
        for sign in (h, -h):
            args = [Q, K, V]
            args[n] = x + sign * d
            side.append(float((ref.forward(law, q, types, cu, *args)[0] * dO).sum()))
        want = (side[0] - side[1]) / (2 * h)
        got = float((grads[n] * d).sum())
        assert abs(got - want) <= 1e-6 * max(1.0, abs(want))
    assert math.isinf(float(lse[0, 5])) and not O[5].any() and not O[20:].any()
