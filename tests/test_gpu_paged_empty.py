"""The paged decode step where a query has no key that counts, and where its
keys count and weigh nothing: zeros in the first case, the formula's 0 / 0 in
the second, whatever the capacity and however the keys are dealt out."""

import pytest
import torch

import attn_ref as ref
from test_gpu_paged import DEV, F32, Cache, P, i32, rnd, stored  # noqa: F401 (P: fixture)

pytestmark = pytest.mark.gpu


def filled(P, kv, K, V, lens, cap, page=16):
    """A cache of the rows K[b], V[b]."""
    Hkv, D = K[0].shape[1:]
    c = Cache(P, kv, Hkv, D, page, len(lens), cap // page)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    P.star_kv_append(c.pages, i32(cu), i32(lens), torch.cat(K).to(DEV), torch.cat(V).to(DEV))
    return c


@pytest.mark.parametrize("cap", [2048, 4096])
@pytest.mark.parametrize("kv", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("lens", [[40, 64, 1, 33], [1500, 64, 20, 700]])
def test_query_of_no_type_over_values_that_are_not_finite(P, kv, cap, lens):
    """Sequences 0 and 1 end in a position of no type: zeros, though their
    keys and values hold infinities and NaN.  The others are as without them."""
    H, Hkv, D, q = 4, 2, 64, 4
    t = ref.cyclic(cap, q)
    t[lens[0] - 1], t[lens[1] - 1] = -1, q
    outs = []
    for odd in (False, True):
        K = [rnd((n, Hkv, D), 10 + b) for b, n in enumerate(lens)]
        V = [rnd((n, Hkv, D), 20 + b) for b, n in enumerate(lens)]
        if odd:
            for b in range(2):
                K[b][:, :, ::3], V[b][:, :, 1::2] = torch.nan, torch.inf
                V[b][::2, :, ::4] = torch.nan
        c = filled(P, kv, K, V, lens, cap)
        outs.append(P.star_attn_decode_paged(P.AttnShape(4, cap, H, Hkv, D, q), c.pages, t.to(DEV), i32(lens),
                                             rnd((4, H, D), 5).to(DEV), out_dtype=F32))
    for O in outs:
        assert not O[:2].any() and bool(torch.isfinite(O).all()) and O[2].any() and O[3].any()
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("cap", [2048, 4096])
@pytest.mark.parametrize("kv", ["bf16", "int8"])
@pytest.mark.parametrize("lens", [[40, 64, 30], [1500, 33, 700]])
def test_keys_that_all_weigh_nothing(P, kv, cap, lens):
    """Every score of one query minus infinity: its softmax is 0 / 0, no
    number, as in the packed forward; not the zeros of a query without keys."""
    H, Hkv, D = 4, 2, 64
    K = [rnd((n, Hkv, D), 10 + b) for b, n in enumerate(lens)]
    V = [rnd((n, Hkv, D), 20 + b) for b, n in enumerate(lens)]
    for x in K:
        x[:, :, 0] = -1.0
    c = filled(P, kv, K, V, lens, cap)
    Q, shape, t = rnd((3, H, D), 5), P.AttnShape(3, cap, H, Hkv, D, 1, "dense"), torch.zeros(cap, dtype=torch.int32)
    O = P.star_attn_decode_paged(shape, c.pages, t.to(DEV), i32(lens), Q.to(DEV), out_dtype=F32)
    for b in range(3):
        Qb = Q.clone()
        Qb[b, 2, 0] = torch.inf
        Ob = P.star_attn_decode_paged(shape, c.pages, t.to(DEV), i32(lens), Qb.to(DEV), out_dtype=F32)
        odd = torch.zeros((3, H), dtype=torch.bool, device=DEV)
        odd[b, 2] = True
        assert bool(torch.isnan(Ob[odd]).all()) and torch.equal(Ob[~odd], O[~odd])


@pytest.mark.parametrize("cap", [2048, 4096])
@pytest.mark.parametrize("first", [True, False])
def test_keys_some_of_which_weigh_nothing(P, cap, first):
    """Scores below the lowest finite number (3e38 times -3e38) in the first
    or the last three quarters of the keys, whole tiles and whole shares of
    them: these have no weight, the others theirs."""
    H, Hkv, D, lens = 2, 1, 64, [1600, 70, 5]
    K = [rnd((n, Hkv, D), 10 + b) for b, n in enumerate(lens)]
    V = [rnd((n, Hkv, D), 20 + b) for b, n in enumerate(lens)]
    for x, n in zip(K, lens):
        x[:, :, 0] = 0
        rows = slice(0, 3 * n // 4) if first else slice(n // 4, n)
        x[rows, :, 0] = -3e38
    Q = rnd((3, H, D), 5)
    Q[:, :, 0] = 3e38
    c = filled(P, "bf16", K, V, lens, cap)
    t = torch.zeros(cap, dtype=torch.int32)
    O = P.star_attn_decode_paged(P.AttnShape(3, cap, H, Hkv, D, 1, "dense"), c.pages, t.to(DEV), i32(lens), Q.to(DEV),
                                 out_dtype=F32)
    rO, mag = ref.decode("dense", 1, t, lens, Q, [stored("bf16", x)[0] for x in K], [stored("bf16", x)[0] for x in V])
    assert ref.off(O, rO, (ref.HALF + ref.SLACK) * mag, False) <= 1


@pytest.mark.parametrize("cap", [64, 4096])
@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_scale_bytes_of_zero(P, kv, cap):
    """Rows with scale byte 0 are zeros, whatever their elements: as after
    clearing a cache's scales."""
    H, Hkv, D, lens = 4, 2, 64, [40, 17]
    K = [rnd((n, Hkv, D), 10 + b) for b, n in enumerate(lens)]
    V = [rnd((n, Hkv, D), 20 + b) for b, n in enumerate(lens)]
    c = filled(P, kv, K, V, lens, cap)
    for b, u in ((0, 0), (0, 39), (1, 5), (1, 16)):
        at = int(c.table[b, u // 16])
        c.ks[at, :, u % 16], c.vs[at, 1, u % 16] = 0, 0
        K[b][u], V[b][u, 1] = 0, 0
    k64, v64 = [stored(kv, x)[0] for x in K], [stored(kv, x)[0] for x in V]
    got = P.star_kv_read(c.pages, i32([0, 40, 57]), i32(lens), 57)
    assert torch.equal(got[0].cpu().double(), torch.cat(k64)) and torch.equal(got[1].cpu().double(), torch.cat(v64))
    Q, t = rnd((2, H, D), 5), ref.cyclic(cap, 4)
    O = P.star_attn_decode_paged(P.AttnShape(2, cap, H, Hkv, D, 4), c.pages, t.to(DEV), i32(lens), Q.to(DEV), out_dtype=F32)
    rO, mag = ref.decode("star", 4, t, lens, Q, k64, v64)
    assert ref.off(O, rO, (ref.HALF + ref.SLACK) * mag, False) <= 1
