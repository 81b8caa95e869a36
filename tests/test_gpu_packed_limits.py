"""Attention over packs at the ends of its range: no rows, the longest sequence,
the most sequences, rows wider than 2^32 bytes from end to end, against the
plain 64-bit forms on sampled rows and heads."""

import pytest
import torch

import attn_ref as ref
from test_gpu_packed import DEV, P  # noqa: F401 (P: fixture)

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
BAR = ref.HALF + ref.SLACK


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def rnd(shape, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.empty(shape, dtype=BF16, device=DEV)
    for rows in x.split(1 << 14):  # (no fp32 copy of the whole)
        rows.copy_(torch.randn(rows.shape, generator=g, device=DEV))
    return x


@pytest.mark.parametrize("n", [0, 3])
def test_no_rows(P, n):
    e = lambda h: torch.empty((0, h, 64), dtype=BF16, device=DEV)
    sh = P.AttnShape(n, 0, 4, 2, 64, 4)
    pack = P.star_attn_pack(4, i32([]), i32([0] * (n + 1)))
    O, lse = P.star_attn_packed_fwd(sh, pack, e(4), e(2), e(2), want_lse=True)
    g = P.star_attn_packed_bwd(sh, pack, e(4), e(4), e(2), e(2), O, lse)
    assert O.shape == (0, 4, 64) and lse.shape == (4, 0) and [x.shape[1] for x in g] == [4, 2, 2]


def check_rows(rows, keys, law, q, t, Q, K, V, dO, O, lse, g):
    """Rows `rows` of O and lse and keys `keys` of dV of one sequence and head."""
    n = t.numel()
    s, _, _ = ref.pair_scores(law, q, Q[rows].double().cpu(), K.double().cpu(), t[rows], t)
    s = s.masked_fill(torch.arange(n)[None, :] > rows[:, None], -torch.inf)
    w, v = torch.softmax(s, -1), V.double().cpu()
    assert ref.off(O[rows.to(DEV)], w @ v, BAR * (w @ v.abs()), False) <= 1
    assert float((lse[rows.to(DEV)].cpu().double() - torch.logsumexp(s, -1)).abs().max()) <= 1e-4
    s, _, _ = ref.pair_scores(law, q, Q.double().cpu(), K[keys].double().cpu(), t, t[keys])
    w = torch.exp(s - lse.cpu().double()[:, None]).masked_fill(torch.arange(n)[:, None] < keys[None, :], 0)
    up = dO.double().cpu()
    assert ref.off(g[2][keys.to(DEV)], w.t() @ up, BAR * (w.t() @ up.abs()), False) <= 1


def test_the_longest_sequence(P):
    T, D, q = 1 << 18, 64, 4
    Q, K, V, dO = (rnd((T, 1, D), k) for k in range(4))
    t = ref.cyclic(T, q)
    sh, pack = P.AttnShape(1, T, 1, 1, D, q), P.star_attn_pack(q, t.to(DEV), i32([0, T]))
    O, lse = P.star_attn_packed_fwd(sh, pack, Q, K, V, out_dtype=F32, want_lse=True)
    g = P.star_attn_packed_bwd(sh, pack, dO, Q, K, V, O, lse, out_dtype=F32)
    check_rows(torch.tensor([0, 1, 127, 131071, T - 2, T - 1]), torch.tensor([0, 5, 131072, T - 1]), "star", q, t,
               Q[:, 0], K[:, 0], V[:, 0], dO[:, 0], O[:, 0], lse[0], [x[:, 0] for x in g])
    assert all(bool(torch.isfinite(x).all()) for x in g)


def test_the_most_sequences(P):
    """16384 sequences of 0 to 31 tokens with sixteen types: every one has its
    own items; the first, the last and some between against 64 bits."""
    n, q, D, H, Hkv = 1 << 14, 16, 128, 2, 1
    lens = [(7 * s) % 32 for s in range(n)]
    lens[0], lens[-1] = 31, 29
    cu = [0]
    for v in lens:
        cu.append(cu[-1] + v)
    T = cu[-1] + 11
    gen = torch.Generator().manual_seed(1)
    t = torch.randint(0, q, (T,), generator=gen).to(torch.int32)
    Q, K, V, dO = rnd((T, H, D), 5), rnd((T, Hkv, D), 6), rnd((T, Hkv, D), 7), rnd((T, H, D), 8)
    sh, pack = P.AttnShape(n, T, H, Hkv, D, q), P.star_attn_pack(q, t.to(DEV), i32(cu))
    O, lse = P.star_attn_packed_fwd(sh, pack, Q, K, V, out_dtype=F32, want_lse=True)
    g = P.star_attn_packed_bwd(sh, pack, dO, Q, K, V, O, lse, out_dtype=F32)
    for s in (0, 1, 2, 777, 4096, 8191, 12345, n - 2, n - 1):
        r = slice(cu[s], cu[s + 1])
        one = [x[r].cpu() for x in (dO, Q, K, V)]
        rO, rl, mag = ref.forward("star", q, t[r], [0, lens[s]], *one[1:])
        assert ref.off(O[r], rO, BAR * mag, False) <= 1
        assert lens[s] == 0 or float((lse[:, r].cpu().double() - rl).abs().max()) <= 1e-4
        rg, bars = ref.backward("star", q, t[r], [0, lens[s]], *one, O[r].cpu(), lse[:, r].cpu())
        for a, b, bar in zip(g, rg, bars):
            assert ref.off(a[r], b, bar, False) <= 1
    assert not O[cu[-1]:].any() and not any(x[cu[-1]:].any() for x in g)
    assert all(bool(torch.isfinite(x).all()) for x in (O, *g))


def test_rows_more_than_32_bits_apart(P):
    """One sequence of 2^18 rows of 66 heads of 128, of which one row in 128 is a
    token: places within the sequence are past 2^32 bytes."""
    T, H, D, q = 1 << 18, 66, 128, 2
    assert T * H * D * 2 > 1 << 32
    at = torch.arange(T // 128) * 128 + 127  # the last row among them
    t = torch.full((T,), -1, dtype=torch.int32)
    t[at] = ref.cyclic(at.numel(), q)
    Q, K, V, dO = (rnd((T, H, D), 20 + k) for k in range(4))
    sh, pack = P.AttnShape(1, T, H, H, D, q), P.star_attn_pack(q, t.to(DEV), i32([0, T]))
    O, lse = P.star_attn_packed_fwd(sh, pack, Q, K, V, want_lse=True)
    g = P.star_attn_packed_bwd(sh, pack, dO, Q, K, V, O, lse)
    d = at.to(DEV)
    for h in (0, 65):
        pick = [x[d, h:h + 1].cpu() for x in (dO, Q, K, V)]
        cu, tt = [0, at.numel()], t[at]
        rO, rl, mag = ref.forward("star", q, tt, cu, *pick[1:])
        assert ref.off(O[d, h:h + 1], rO, BAR * mag, True) <= 1
        assert float((lse[h, d].cpu().double() - rl[0]).abs().max()) <= 1e-4
        rg, bars = ref.backward("star", q, tt, cu, *pick, O[d, h:h + 1].cpu(), lse[h:h + 1, d].cpu())
        for a, b, bar in zip(g, rg, bars):
            assert ref.off(a[d, h:h + 1], b, bar, True) <= 1
    empty = torch.tensor([0, 126, 128, T - 2], device=DEV)
    assert not O[empty].any() and not any(x[empty].any() for x in g)
