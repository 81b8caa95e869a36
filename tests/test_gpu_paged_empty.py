"""The paged decode step where a query has no key that counts: zeros, whatever
the capacity and however the keys are dealt out."""

import pytest
import torch

import attn_ref as ref
from test_gpu_paged import DEV, F32, Cache, P, i32, rnd  # noqa: F401 (P: fixture)

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
