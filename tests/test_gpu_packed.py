"""Attention over packs and its gradient on the GPU against the plain 64-bit
forms of attn_ref (whose docstring derives the bars): lengths from none to
several blocks, both head widths, group widths 8 to 128, every law, grouped
heads, rows of a type out of range, rows behind the last sequence."""

import pytest
import torch

import attn_ref as ref

pytestmark = pytest.mark.gpu

DEV, BF16, F32 = "cuda", torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU parity tests need a GPU"
    import paper_2609_32814_amd as P
    return P


def starts(lens, first=0):
    cu = [first]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


class Pack:
    """Inputs of a pack on the CPU, and its calls on the GPU."""

    def __init__(self, P, law, q, D, H, Hkv, lens, seed=0, tail=0, first=0, types=None):
        g = torch.Generator().manual_seed(1000 * seed + sum(lens) + 7 * D + q)
        self.P, self.law, self.q, self.cu = P, law, q, starts(lens, first)
        self.T = self.cu[-1] + tail
        rnd = lambda h: torch.randn((self.T, h, D), generator=g).to(BF16)
        self.Q, self.K, self.V, self.dO = rnd(H), rnd(Hkv), rnd(Hkv), rnd(H)
        pos = [torch.arange(n) for n in lens]
        self.types = torch.full((self.T,), -1, dtype=torch.int32)
        self.types[first:self.cu[-1]] = torch.cat([(p % q) for p in pos]).to(torch.int32) if lens else 0
        if types == "random":
            self.types[:] = torch.randint(0, q, (self.T,), generator=g).to(torch.int32)
        elif types == "interval":
            self.types[first:self.cu[-1]] = torch.cat([(p // 40) % q for p in pos]).to(torch.int32)
        elif types == "some_bad":
            bad = torch.rand((self.T,), generator=g) < 0.3
            self.types[bad] = torch.tensor([-1, q, 1 << 20], dtype=torch.int32)[torch.randint(0, 3, (int(bad.sum()),))]
        self.shape = P.AttnShape(len(lens), self.T, H, Hkv, D, q, law)
        self.d = {k: getattr(self, k).to(DEV) for k in ("Q", "K", "V", "dO", "types")}
        self.dcu = torch.tensor(self.cu, dtype=torch.int32, device=DEV)
        self.pack = P.star_attn_pack(q, self.d["types"], self.dcu)

    def fwd(self, **kw):
        return self.P.star_attn_packed_fwd(self.shape, self.pack, self.d["Q"], self.d["K"], self.d["V"], **kw)

    def bwd(self, O, lse, **kw):
        return self.P.star_attn_packed_bwd(self.shape, self.pack, self.d["dO"], self.d["Q"], self.d["K"], self.d["V"],
                                           O, lse, **kw)

    def check(self, out_dtype=F32):
        O, lse = self.fwd(out_dtype=out_dtype, want_lse=True)
        rO, rl, mag = ref.forward(self.law, self.q, self.types, self.cu, self.Q, self.K, self.V)
        assert ref.off(O, rO, (ref.HALF + ref.SLACK) * mag, out_dtype == BF16) <= 1
        got = lse.cpu().double()
        seen = torch.isfinite(rl)
        assert torch.equal(torch.isneginf(got), ~seen)
        assert not seen.any() or float((got[seen] - rl[seen]).abs().max()) <= 1e-4
        g = self.bwd(O, lse, out_dtype=out_dtype)
        # (lse of rows without a key is -inf on both sides and not read)
        rg, bars = ref.backward(self.law, self.q, self.types, self.cu, self.dO, self.Q, self.K, self.V, O.cpu(), lse.cpu())
        for name, a, b, bar in zip(("dQ", "dK", "dV"), g, rg, bars):
            assert ref.off(a, b, bar, out_dtype == BF16) <= 1, name
        return O, lse, g


# (law, q, head_dim, n_heads, n_kv, lengths, types)
CASES = [
    ("star", 1, 64, 1, 1, [1], None),
    ("star", 4, 64, 2, 2, [1, 1, 1], None),
    ("star", 4, 64, 2, 2, [0, 5, 0, 0, 3, 0], None),
    ("dense", 1, 64, 3, 3, [64, 65, 63], None),
    ("dense", 1, 128, 4, 2, [127, 128, 129], None),
    ("dense", 4, 64, 2, 1, [130, 31], None),
    ("star", 2, 64, 4, 2, [300, 1, 77], None),
    ("star", 4, 64, 12, 12, [33, 210], None),
    ("tensor2", 4, 64, 2, 1, [515, 40], "interval"),
    ("tensor2", 2, 128, 2, 2, [90, 200], None),
    ("star", 8, 64, 2, 2, [190, 66], "random"),       # groups of 8 features
    ("star", 16, 128, 2, 2, [160, 17], None),
    ("star", 8, 128, 4, 1, [260], "random"),
    ("star", 4, 128, 8, 1, [333, 2], "random"),       # eight query heads on one
    ("star", 2, 128, 6, 2, [700], None),
    ("star", 4, 64, 3, 1, [1025], "random"),
    # many heads: one group of wavefronts per work item, and the star law's
    # kernels that leave feature blocks out
    ("dense", 1, 64, 224, 224, [200, 77], None),
    ("tensor2", 4, 64, 144, 144, [330], "interval"),
    ("star", 2, 64, 160, 160, [150, 1], "random"),
    ("star", 4, 64, 96, 96, [150, 99], "random"),
    ("star", 8, 64, 96, 96, [190], "random"),
    ("star", 4, 64, 192, 96, [170, 40], None),
    ("dense", 1, 128, 64, 64, [140, 70], None),
    ("star", 2, 128, 64, 16, [200, 33], None),
    ("star", 4, 128, 64, 64, [150, 130], "random"),
    ("star", 4, 128, 64, 8, [260, 2], None),
    ("star", 8, 128, 64, 64, [170, 65], "random"),
    ("star", 16, 128, 64, 64, [260], "random"),
    ("star", 4, 64, 72, 72, [140, 50, 9], "some_bad"),
    ("star", 4, 64, 2, 2, [140, 50, 9], "some_bad"),
    # query heads of a key/value head dealt to several work items
    ("star", 4, 64, 8, 2, [140, 50, 9], "some_bad"),
    ("dense", 1, 128, 16, 2, [100, 0, 131], None),
    ("tensor2", 4, 64, 12, 1, [300, 77], "interval"),
    ("dense", 1, 128, 2, 2, [100, 3], "some_bad"),
]


def _id(c):
    return f"{c[0]}-q{c[1]}-d{c[2]}-h{c[3]}/{c[4]}-{'+'.join(map(str, c[5]))}-{c[6] or 'cyclic'}"


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_forward_and_gradient(P, case):
    law, q, D, H, Hkv, lens, types = case
    Pack(P, law, q, D, H, Hkv, lens, types=types).check()


def test_bf16_results(P):
    Pack(P, "star", 4, 64, 4, 2, [150, 70], seed=3).check(BF16)
    Pack(P, "star", 2, 128, 4, 4, [150, 70], seed=3).check(BF16)


def test_long_sequence_against_sampled_rows(P):
    """A sequence of 9000 beside short ones: rows of one head, the last ones
    and some between, and the whole gradient of the last keys' values."""
    p = Pack(P, "star", 4, 64, 2, 1, [70, 9000, 5], seed=5)
    O, lse = p.fwd(out_dtype=F32, want_lse=True)
    a, rows = 70, torch.tensor([0, 63, 64, 4095, 8191, 8998, 8999])
    t = p.types[70:9070]
    for h in range(2):
        s, _, _ = ref.pair_scores("star", 4, p.Q[a + rows, h].double(), p.K[a:a + 9000, 0].double(), t[rows], t)
        s = s.masked_fill(torch.arange(9000)[None, :] > rows[:, None], -torch.inf)
        w, V = torch.softmax(s, -1), p.V[a:a + 9000, 0].double()
        assert ref.off(O[a + rows.to(DEV), h], w @ V, (ref.HALF + ref.SLACK) * (w @ V.abs()), False) <= 1
        assert float((lse[h, a + rows.to(DEV)].cpu().double() - torch.logsumexp(s, -1)).abs().max()) <= 1e-4
    g = p.bwd(O, lse, out_dtype=F32)
    # one probability vector per query in the formula: dV of sampled keys
    u = torch.tensor([0, 1, 4500, 8999])
    dV, bar = torch.zeros((4, 64), dtype=ref.F64), torch.zeros((4, 64), dtype=ref.F64)
    for h in range(2):
        s, _, _ = ref.pair_scores("star", 4, p.Q[a:a + 9000, h].double(), p.K[a + u, 0].double(), t, t[u])
        w = torch.exp(s - lse[h, a:a + 9000].cpu().double()[:, None]).masked_fill(torch.arange(9000)[:, None] < u[None, :], 0)
        dV += w.t() @ p.dO[a:a + 9000, h].double()
        bar += (ref.HALF + ref.SLACK) * (w.t() @ p.dO[a:a + 9000, h].double().abs())
    assert ref.off(g[2][a + u.to(DEV), 0], dV, bar, False) <= 1
    assert all(bool(torch.isfinite(x).all()) for x in g)


def test_rows_outside_every_sequence(P):
    """The caller's rows before the first and behind the last sequence are
    left as they were; in buffers that a call allocates they are zeros."""
    p = Pack(P, "star", 4, 64, 4, 2, [50, 90], tail=300, first=7)
    out = torch.ones(p.T, dtype=torch.bool, device=DEV)
    out[7:147] = False
    O, lse, g = p.check()
    for x in (O, *g):
        assert not x[out].any()
    own = [torch.full_like(x, 7.5) for x in (O, *g)]
    lse2 = torch.full_like(lse, 7.5)
    p.fwd(O=own[0], lse=lse2)
    p.bwd(own[0], lse2, dQ=own[1], dK=own[2], dV=own[3])
    for a, b in zip(own, (O, *g)):
        assert bool((a[out] == 7.5).all()) and torch.equal(a[~out], b[~out])
    assert bool((lse2[:, out] == 7.5).all()) and torch.equal(lse2[:, ~out], lse[:, ~out])
    # no sequence at all
    e = Pack(P, "star", 2, 64, 2, 2, [], tail=20)
    assert not e.fwd().any()


def test_bounds_that_cannot_be_are_cut(P):
    """Bounds that decrease or leave the rows count as the nearest allowed:
    here as [0, 60, 60, 200]."""
    good = Pack(P, "star", 2, 64, 2, 2, [60, 0, 140])
    odd = torch.tensor([-5, 60, 40, 5000], dtype=torch.int32, device=DEV)
    pack = P.star_attn_pack(2, good.d["types"], odd)
    O = P.star_attn_packed_fwd(good.shape, pack, good.d["Q"], good.d["K"], good.d["V"])
    assert torch.equal(O, good.fwd())


def test_pack_of_another_shape_writes_nothing(P):
    a = Pack(P, "star", 2, 64, 2, 2, [60, 40])
    b = Pack(P, "star", 2, 64, 2, 2, [50, 30, 20])  # T alike, another count of sequences
    big = torch.zeros(max(a.pack.numel(), b.pack.numel()), dtype=torch.uint8, device=DEV)
    big[:b.pack.numel()] = b.pack
    O = torch.full((a.T, 2, 64), 3.0, dtype=F32, device=DEV)
    P.star_attn_packed_fwd(a.shape, big, a.d["Q"], a.d["K"], a.d["V"], O=O)
    assert bool((O == 3.0).all())


def test_equal_lengths_match_the_batched_forward(P):
    """Two sequences of equal length: the pack's rows and those of
    star_attn_fwd are each within their bar of one 64-bit result."""
    B, S, H, Hkv, D, q = 2, 257, 4, 2, 128, 2
    p = Pack(P, "star", q, D, H, Hkv, [S, S], seed=9)
    plan = P.star_type_plan(q, ref.cyclic(S, q).to(DEV))
    v = lambda x: p.d[x].view(B, S, -1, D)
    O, lse = P.star_attn_fwd(P.AttnShape(B, S, H, Hkv, D, q), plan, v("Q"), v("K"), v("V"), out_dtype=F32, want_lse=True)
    Op, lp = p.fwd(out_dtype=F32, want_lse=True)
    rO, rl, mag = ref.forward("star", q, p.types, p.cu, p.Q, p.K, p.V)
    for x in (O.view(B * S, H, D), Op):
        assert ref.off(x, rO, (ref.HALF + ref.SLACK) * mag, False) <= 1
    for x in (lse.permute(1, 0, 2).reshape(H, B * S), lp):
        assert float((x.cpu().double() - rl).abs().max()) <= 1e-4


def test_repeated_calls_are_equal(P):
    p = Pack(P, "star", 4, 64, 6, 2, [700, 90, 300], types="random", seed=2)
    O, lse = p.fwd(want_lse=True)
    first = (O, lse, *p.bwd(O, lse))
    for _ in range(3):
        p.pack = P.star_attn_pack(4, p.d["types"], p.dcu)
        O, lse = p.fwd(want_lse=True)
        for a, b in zip(first, (O, lse, *p.bwd(O, lse))):
            assert torch.equal(a, b)


def test_one_token_sequences_have_no_score_gradient(P):
    """With one key P = 1 and dP = delta up to rounding of O: with O in fp32
    dQ and dK vanish to fp32 rounding, and dV is dO."""
    p = Pack(P, "star", 4, 64, 4, 4, [1] * 37)
    O, lse = p.fwd(out_dtype=F32, want_lse=True)
    dQ, dK, dV = p.bwd(O, lse, out_dtype=F32)
    lim = 2.0 ** -18 * float((p.dO.double().abs() * p.V.double().abs()).sum(-1).max()) * 4
    assert float(dQ.abs().max()) <= lim and float(dK.abs().max()) <= lim
    assert float((dV.cpu().double() - p.dO.double()).abs().max()) <= 2.0 ** -8 * float(p.dO.abs().max())


def test_side_stream_and_graph_replays(P):
    """Plan, forward and gradient on a stream of their own, captured, replayed
    with other rows and other bounds, against eager calls."""
    a = Pack(P, "star", 4, 64, 4, 2, [90, 110], seed=11)
    b = Pack(P, "star", 4, 64, 4, 2, [13, 187], seed=12, types="random")
    d = {k: v.clone() for k, v in a.d.items()}
    cu, pack = a.dcu.clone(), torch.empty_like(a.pack)
    ws = torch.empty(P.star_attn_packed_bwd_workspace_bytes(a.shape), dtype=torch.uint8, device=DEV)

    def step():
        P.star_attn_pack(4, d["types"], cu, pack=pack)
        O, lse = P.star_attn_packed_fwd(a.shape, pack, d["Q"], d["K"], d["V"], want_lse=True)
        return (O, lse, *P.star_attn_packed_bwd(a.shape, pack, d["dO"], d["Q"], d["K"], d["V"], O, lse, ws=ws))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        warm = step()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        outs = step()
    for src in (a, b, a, b):
        for k in d:
            d[k].copy_(src.d[k])
        cu.copy_(src.dcu)
        g.replay()
        torch.cuda.synchronize()
        O, lse = src.fwd(want_lse=True)
        for x, y in zip(outs, (O, lse, *src.bwd(O, lse))):
            assert torch.equal(x, y)
    assert torch.equal(warm[0], a.fwd())


ODD = [
    ("dense", 1, 64, 2, 2, [150, 70], None),
    ("star", 4, 64, 2, 1, [200, 30], "random"),
    ("tensor2", 2, 128, 4, 2, [140, 31], None),
    ("star", 4, 64, 96, 96, [160, 40], None),
    ("star", 4, 128, 64, 16, [170], "random"),
    ("dense", 1, 128, 64, 64, [140], None),
    ("star", 2, 64, 6, 2, [131], "some_bad"),
]


@pytest.mark.parametrize("law,q,D,H,Hkv,lens,types", ODD)
@pytest.mark.parametrize("t", [0, 37, 129])
def test_what_is_not_finite_stays_out_of_masked_places(P, law, q, D, H, Hkv, lens, types, t):
    """A position with infinities and NaN reaches neither the earlier positions
    of its sequence nor another sequence: their weights of it are none, and
    not zero times it.  Values of V that are infinite or NaN reach their own
    feature alone."""
    c = Pack(P, law, q, D, H, Hkv, lens, seed=5, types=types)
    c.types[t] = 0
    c.d["types"] = c.types.to(DEV)
    c.pack = P.star_attn_pack(q, c.d["types"], c.dcu)
    keep = torch.ones(c.T, dtype=torch.bool)
    keep[t:lens[0]] = False  # rows that may not see position t
    O, lse = c.fwd(out_dtype=F32, want_lse=True)
    rO, rl, mag = ref.forward(law, q, c.types, c.cu, c.Q, c.K, c.V)
    bar = (ref.HALF + ref.SLACK) * mag

    # V: features 3 (infinite), 20 (minus), 21 (NaN)
    V = c.V.clone()
    V[t, :, 3], V[t, :, 20], V[t, :, 21] = torch.inf, -torch.inf, torch.nan
    c.d["V"] = V.to(DEV)
    O1, l1 = c.fwd(out_dtype=F32, want_lse=True)
    rest = [f for f in range(D) if f not in (3, 20, 21)]
    assert ref.off(O1[:, :, rest], rO[:, :, rest], bar[:, :, rest], False) <= 1
    assert ref.off(O1[keep.to(DEV)], rO[keep], bar[keep], False) <= 1
    assert torch.equal(l1, lse)
    hit = (~keep & ref.valid(c.types, q)).to(DEV)
    assert bool(torch.isposinf(O1[hit][:, :, 3]).all()) and bool(torch.isneginf(O1[hit][:, :, 20]).all())
    assert bool(torch.isnan(O1[hit][:, :, 21]).all())

    # K too: dQ of the rows that do not see it
    K = c.K.clone()
    K[t, :, ::5], K[t, :, 1::5] = torch.nan, torch.inf
    c.d["K"] = K.to(DEV)
    O2, l2 = c.fwd(out_dtype=F32, want_lse=True)
    assert ref.off(O2[keep.to(DEV)], rO[keep], bar[keep], False) <= 1
    dQ = c.bwd(O2, l2, out_dtype=F32)[0]
    ko, kl = keep[:, None, None], keep[None, :]
    rg, bars = ref.backward(law, q, c.types, c.cu, c.dO, c.Q, c.K, c.V, torch.where(ko, O2.cpu(), O.cpu()),
                            torch.where(kl, l2.cpu(), lse.cpu()))
    assert ref.off(dQ[keep.to(DEV)], rg[0][keep], bars[0][keep], False) <= 1

    # Q and dO: dK and dV of the keys that it does not see
    c.d["K"], c.d["V"] = c.K.to(DEV), c.V.to(DEV)
    Q, dO = c.Q.clone(), c.dO.clone()
    Q[t, :, ::5], Q[t, :, 1::5] = torch.nan, torch.inf
    dO[t, :, 2::3] = -torch.inf
    c.d["Q"], c.d["dO"] = Q.to(DEV), dO.to(DEV)
    O3, l3 = c.fwd(out_dtype=F32, want_lse=True)
    behind = torch.ones(c.T, dtype=torch.bool)
    behind[:t + 1] = False
    own = torch.arange(c.T) != t
    _, dK, dV = c.bwd(O3, l3, out_dtype=F32)
    rg, bars = ref.backward(law, q, c.types, c.cu, c.dO, c.Q, c.K, c.V, torch.where(own[:, None, None], O3.cpu(), O.cpu()),
                            torch.where(own[None, :], l3.cpu(), lse.cpu()))
    assert ref.off(dK[behind.to(DEV)], rg[1][behind], bars[1][behind], False) <= 1
    assert ref.off(dV[behind.to(DEV)], rg[2][behind], bars[2][behind], False) <= 1


def test_a_query_that_is_no_number(P):
    """A row of Q with a NaN, or with infinities on both sides of a product:
    NaN in its own row of O and lse alone."""
    for D, H in ((64, 2), (64, 96), (128, 3)):
        c = Pack(P, "dense", 1, D, H, H, [70, 150], seed=2)
        O, lse = c.fwd(out_dtype=F32, want_lse=True)
        Q = c.Q.clone()
        Q[3, :, 5] = torch.nan
        Q[100, :, 0], Q[100, :, 1] = torch.inf, -torch.inf
        c.d["Q"] = Q.to(DEV)
        O1, l1 = c.fwd(out_dtype=F32, want_lse=True)
        odd = torch.zeros(c.T, dtype=torch.bool, device=DEV)
        odd[3] = odd[100] = True
        assert bool(torch.isnan(O1[3]).all()) and bool(torch.isnan(l1[:, 3]).all())
        assert not bool(torch.isfinite(O1[100]).any()) and not bool(torch.isfinite(l1[:, 100]).any())
        assert torch.equal(O1[~odd], O[~odd]) and torch.equal(l1[:, ~odd], lse[:, ~odd])


def test_lse_of_rows_outside_every_sequence(P):
    c = Pack(P, "star", 2, 64, 2, 2, [40, 9], seed=3, tail=300, first=5)
    rest = torch.ones(c.T, dtype=torch.bool, device=DEV)
    rest[5:54] = False
    O = torch.full((c.T, 2, 64), 7.0, device=DEV)
    _, lse = c.fwd(O=O, want_lse=True)
    assert bool(torch.isneginf(lse[:, rest]).all()) and bool(torch.isfinite(lse[:, ~rest]).all()) and bool((O[rest] == 7).all())
    own = torch.full((2, c.T), 3.0, device=DEV)
    c.fwd(O=O, lse=own)
    assert bool((own[:, rest] == 3).all()) and torch.equal(own[:, ~rest], lse[:, ~rest])
    O2, lse2 = c.fwd(lse=own, out_dtype=F32)
    assert not O2[rest].any() and bool(torch.isneginf(lse2[:, rest]).all()) and torch.equal(O2[~rest], O[~rest])


@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_gradient_sums_of_dealt_heads(P, out_dtype):
    """Where heads are dealt: rows outside the sequences stay, rows of a type out
    of range are zeros, a repeated call gives the same bits."""
    c = Pack(P, "star", 4, 128, 8, 1, [90, 60], seed=9, tail=70, first=3, types="some_bad")
    O, lse = c.fwd(out_dtype=F32, want_lse=True)
    got = []
    for _ in range(2):
        g = [torch.full((c.T, h, 128), 7.0, dtype=out_dtype, device=DEV) for h in (8, 1, 1)]
        c.bwd(O, lse, dQ=g[0], dK=g[1], dV=g[2])
        got.append(g)
    ok = ref.valid(c.types, 4)
    inside = torch.zeros(c.T, dtype=torch.bool)
    inside[3:153] = True
    rg, bars = ref.backward("star", 4, c.types, c.cu, c.dO, c.Q, c.K, c.V, O.cpu(), lse.cpu())
    for a, b, r, bar in zip(got[0], got[1], rg, bars):
        assert torch.equal(a, b)
        a = a.cpu()
        assert bool((a[~inside] == 7).all()) and not a[inside & ~ok].any()
        assert ref.off(a[inside], r[inside], bar[inside], out_dtype == BF16) <= 1


def test_two_streams_share_a_pack(P):
    """Forward and gradient on two streams at once, one pack between them."""
    a = Pack(P, "star", 4, 64, 8, 2, [300, 170, 5], seed=1)
    b = Pack(P, "star", 4, 64, 8, 2, [300, 170, 5], seed=2)
    want = []
    for c in (a, b):
        O, lse = c.fwd(want_lse=True)
        want.append([O, lse, *c.bwd(O, lse)])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(4):
        for k, c in enumerate((a, b)):
            with torch.cuda.stream(streams[k]):
                c.pack = a.pack
                O, lse = c.fwd(want_lse=True)
                got[k].append([O, lse, *c.bwd(O, lse)])
    torch.cuda.synchronize()
    for k in range(2):
        for g in got[k]:
            assert all(torch.equal(x, y) for x, y in zip(g, want[k]))
