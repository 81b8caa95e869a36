"""The paged cache's calls on bounds of sequences that cannot be: each counts
as the nearest that is allowed, as in a pack's plan, so that one array names
the same rows to every call."""

import pytest
import torch

from test_gpu_paged import DEV, Cache, P, i32, rnd, stored  # noqa: F401 (P: fixture)

pytestmark = pytest.mark.gpu


def allowed(cu, T):
    """The bounds that `cu` counts as: no lower than an earlier one or 0, no
    higher than T."""
    out, top = [], 0
    for v in cu:
        top = max(top, v)
        out.append(min(top, T))
    return out


ODD = [
    ([-5, 60, 40, 5000], 200),
    ([0, 100], 64),                       # one sequence, an end past the rows
    ([0, 10, 5, 20, 30], 30),
    ([0, 10, 50, 20], 50),                # a last bound below an earlier one
    ([7, 3, 3, 40, 1], 41),
    ([500, 0, 5], 20),                    # no row is left
    ([0, -2 ** 31, 2 ** 31 - 1, 4], 33),
]


def both(P, kv, cu, T, Hkv, D, page, length, seed=0):
    """Append and read with `cu` and with what it counts as: (caches, rows
    read, rows read into the caller's)."""
    B, cap = len(cu) - 1, -(-max(length) // page)
    K, V = rnd((T, Hkv, D), 1 + seed).to(DEV), rnd((T, Hkv, D), 2 + seed).to(DEV)
    out = []
    for bounds in (cu, allowed(cu, T)):
        c = Cache(P, kv, Hkv, D, page, B, cap, seed=seed)
        P.star_kv_append(c.pages, i32(bounds), i32(length), K, V)
        own = [torch.full_like(K, 5.0), torch.full_like(V, 5.0)]
        P.star_kv_read(c.pages, i32(bounds), i32(length), T, *own)
        held = [x.view(torch.uint8) for x in (c.K, c.V, c.ks, c.vs) if x is not None]
        out.append((*held, *P.star_kv_read(c.pages, i32(bounds), i32(length), T), *own))
    return out


@pytest.mark.parametrize("kv", ["bf16", "int8"])
@pytest.mark.parametrize("cu,T", ODD)
def test_bounds_that_cannot_be_are_cut(P, kv, cu, T):
    length = [max(1, T // 2 + 3 * b) for b in range(len(cu) - 1)]
    for a, b in zip(*both(P, kv, cu, T, 2, 64, 8, length)):
        assert torch.equal(a, b)


# (several rounds of bounds per wavefront, 4 and 16 tokens a workgroup)
@pytest.mark.parametrize("B,T", [(300, 700), (1500, 900), (4500, 5000)])
def test_many_sequences_with_bounds_out_of_order(P, B, T):
    g = torch.Generator().manual_seed(B)
    cu = torch.sort(torch.randint(0, T + 1, (B + 1,), generator=g)).values
    odd = torch.rand((B + 1,), generator=g) < 0.2
    cu[odd] += torch.randint(-40, 9, (int(odd.sum()),), generator=g)
    cu = cu.tolist()
    assert cu != allowed(cu, T)
    length = torch.randint(0, 60, (B,), generator=g).tolist()
    for a, b in zip(*both(P, "bf16", cu, T, 1, 64, 16, length, seed=3)):
        assert torch.equal(a, b)
    # and in order, against the rows themselves: what has a place is read back
    cu = allowed(cu, T)
    c = Cache(P, "bf16", 1, 64, 16, B, 4, seed=4)
    K = rnd((T, 1, 64), 5)
    P.star_kv_append(c.pages, i32(cu), i32(length), K.to(DEV), K.to(DEV))
    want = torch.zeros_like(K)
    for b in range(B):
        for t in range(cu[b], cu[b + 1]):
            if length[b] - (cu[b + 1] - t) >= 0:
                want[t] = K[t]
    for x in P.star_kv_read(c.pages, i32(cu), i32(length), T):
        assert torch.equal(x.cpu(), want)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_no_sequence_at_all(P, kv):
    """A cache of no sequences: every row is outside, none is written, all are
    read back as zeros or left as they were."""
    c = Cache(P, kv, 2, 64, 8, 0, 3)
    before = [x.view(torch.uint8).clone() for x in (c.K, c.V)]
    K = rnd((5, 2, 64), 1).to(DEV)
    P.star_kv_append(c.pages, i32([0]), i32([]), K, K)
    assert all(torch.equal(a, b.view(torch.uint8)) for a, b in zip(before, (c.K, c.V)))
    assert not any(x.any() for x in P.star_kv_read(c.pages, i32([0]), i32([]), 5))
    own = [torch.full_like(K, 5.0) for _ in range(2)]
    P.star_kv_read(c.pages, i32([3]), i32([]), 5, *own)
    assert all(bool((x == 5).all()) for x in own)
    assert P.star_kv_read(c.pages, i32([0]), i32([]), 0)[0].shape == (0, 2, 64)
    O = P.star_attn_decode_paged(P.AttnShape(0, 24, 2, 2, 64, 1), c.pages, i32([0] * 24), i32([]), K[:0])
    assert O.shape == (0, 2, 64)


def test_sequences_share_pages(P):
    """Two sequences with one prompt's pages in both tables, going on in pages
    of their own: each reads the whole of its own positions."""
    D, Hkv, page = 64, 2, 8
    c = Cache(P, "int8", Hkv, D, page, 2, 4)
    c.dtable[1, :2] = c.dtable[0, :2]
    K = [rnd((n, Hkv, D), 3 + k).to(DEV) for k, n in enumerate((16, 5, 9))]
    P.star_kv_append(c.pages, i32([0, 16, 16]), i32([16, 0]), K[0], K[0])
    P.star_kv_append(c.pages, i32([0, 5, 14]), i32([21, 25]), torch.cat(K[1:]), torch.cat(K[1:]))
    got = P.star_kv_read(c.pages, i32([0, 21, 46]), i32([21, 25]), 46)
    want = torch.cat([stored("int8", x.cpu())[0] for x in (K[0], K[1], K[0], K[2])])
    for x in got:
        assert torch.equal(x.cpu().double(), want)
