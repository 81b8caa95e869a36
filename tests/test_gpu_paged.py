"""The paged cache and its decode step on the GPU against plain 64-bit forms:
page sizes from 8, tables in any order, lengths from none to several tiles,
8-bit rows bit for bit, pages that are not there, offsets past 32 bits."""

import pytest
import torch

import attn_ref as ref

pytestmark = pytest.mark.gpu

DEV, BF16, F32, F64 = "cuda", torch.bfloat16, torch.float32, torch.float64
TYPES = {"bf16": BF16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"e4m3": 448.0, "int8": 127.0}


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU parity tests need a GPU"
    import paper_2609_32814_amd as P
    return P


def stored(kv, x):
    """(values in 64 bits, scale bytes) that rows [..., D] are kept as."""
    x = x.to(F64)
    if kv == "bf16":
        return x, None
    top = x.abs().amax(-1, keepdim=True)
    e = torch.full(top.shape, -126)
    for k in range(-126, 128):
        e = torch.where(top > TOP[kv] * 2.0 ** k, k + 1, e)
    up = torch.ldexp(torch.ones_like(top), e)
    y = x / up
    y = y.to(F32).to(torch.float8_e4m3fn).to(F64) if kv == "e4m3" else torch.round(y)
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    vals = torch.where(bad, torch.full_like(x, torch.nan), y * up)
    return vals, torch.where(bad, 255, e + 127)[..., 0].to(torch.uint8)


class Cache:
    """A paged cache on the GPU, its table in a random order."""

    def __init__(self, P, kv, Hkv, D, page, B, max_pages, spare=2, seed=0):
        g = torch.Generator().manual_seed(seed + 13 * page)
        self.kv, self.n = kv, B * max_pages + spare
        shape = (self.n, Hkv, page, D)
        fill = (lambda: torch.full(shape, 1.5, dtype=BF16, device=DEV)) if kv == "bf16" else \
            (lambda: torch.full(shape, 0x11, dtype=torch.uint8, device=DEV).view(TYPES[kv]))
        self.K, self.V = fill(), fill()
        scale = lambda: None if kv == "bf16" else torch.full(shape[:3], 120, dtype=torch.uint8, device=DEV)
        self.ks, self.vs = scale(), scale()
        self.table = torch.randperm(self.n, generator=g)[:B * max_pages].view(B, max_pages).to(torch.int32)
        self.dtable = self.table.to(DEV)
        self.pages = P.KVPages(self.K, self.V, self.dtable, self.ks, self.vs)


def rnd(shape, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(BF16)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("kv", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("D,Hkv,page", [(64, 3, 8), (128, 2, 32), (128, 1, 16)])
def test_append_and_read(P, kv, D, Hkv, page):
    """Prompts of 0, 1, 37 and 21 tokens, then a step of one token each and a
    step that leaves some out: what is read back is what the rows stand for,
    bit for bit, and no other place changes."""
    B, cap = 4, 64
    c = Cache(P, kv, Hkv, D, page, B, cap // page)
    before = [x.clone().view(torch.uint8) for x in (c.K, c.V)]
    held = [torch.zeros((0, Hkv, D), dtype=F64) for _ in range(2 * B)]
    length = [0] * B
    for step, add in enumerate([[0, 1, 37, 21], [1, 1, 1, 1], [0, 3, 0, 1]]):
        cu = [0]
        for n in add:
            cu.append(cu[-1] + n)
        length = [a + n for a, n in zip(length, add)]
        K, V = rnd((cu[-1], Hkv, D), 40 + step), rnd((cu[-1], Hkv, D), 50 + step, 1e-3)
        K[0, 0] = 0          # a row of zeros
        V[0, 0, :] = 2.0 ** -130  # below the smallest scale
        P.star_kv_append(c.pages, i32(cu), i32(length), K.to(DEV), V.to(DEV))
        for x, rows in enumerate((K, V)):
            vals, _ = stored(kv, rows)
            for b in range(B):
                held[B * x + b] = torch.cat([held[B * x + b], vals[cu[b]:cu[b + 1]]])
        all_cu = [0]
        for n in length:
            all_cu.append(all_cu[-1] + n)
        got = P.star_kv_read(c.pages, i32(all_cu), i32(length), all_cu[-1])
        for x in range(2):
            assert torch.equal(got[x].cpu().to(F64), torch.cat(held[B * x:B * x + B]))
    # places that hold no position are as they were
    used = torch.zeros((c.n, page), dtype=torch.bool)
    for b in range(B):
        pos = torch.arange(length[b])
        used[c.table[b, pos // page].long(), pos % page] = True
    for x, old in zip((c.K, c.V), before):
        now = x.view(torch.uint8).cpu().permute(0, 2, 1, 3)
        assert torch.equal(now[~used], old.cpu().permute(0, 2, 1, 3)[~used])


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_scales_borders_and_rows_that_are_not_finite(P, kv):
    """Largest magnitudes at, just below and just above a power of two times
    the type's top, ties between two steps, and rows with a NaN or infinity."""
    D, top = 64, TOP[kv]
    tops = [top, top * (1 - 2.0 ** -8), top * (1 + 2.0 ** -7), 1.0, 1.75, 1.7578125, 1.984375, 1.9921875, 3e38, 2.0 ** -126,
            2.0 ** -133]
    K = torch.zeros((len(tops) + 3, 1, D))
    for r, t in enumerate(tops):
        K[r, 0] = torch.linspace(-1, 1, D) * t
    K[-3, 0, 5], K[-2, 0, 6], K[-1, 0, 7] = torch.nan, torch.inf, -torch.inf
    K = K.to(BF16)
    T = K.shape[0]
    c = Cache(P, kv, 1, D, 8, 1, 4)
    P.star_kv_append(c.pages, i32([0, T]), i32([T]), K.to(DEV), K.to(DEV))
    want, scale = stored(kv, K)
    for x, s in zip(P.star_kv_read(c.pages, i32([0, T]), i32([T]), T), (c.ks, c.vs)):
        x = x.cpu().to(F64)
        assert torch.equal(torch.isnan(x), torch.isnan(want)) and int(torch.isnan(x).sum()) == 3 * D
        assert torch.equal(torch.nan_to_num(x), torch.nan_to_num(want))
        pos = torch.arange(T)
        assert torch.equal(s.cpu()[c.table[0, pos // 8].long(), 0, pos % 8], scale[:, 0])


def test_rows_that_have_no_place(P):
    """Pages out of range, positions past the capacity or below zero, rows of
    no sequence: not written; read back as zeros or left as they were."""
    D, page, T = 64, 8, 30
    c = Cache(P, "int8", 2, D, page, 2, 2)
    c.dtable[0, 1], c.dtable[1, 0] = c.n, -1
    K = rnd((T, 2, D), 1)
    before = [x.clone() for x in (c.K, c.V, c.ks, c.vs)]
    # sequence 0: positions 4 .. 15 of rows 3 .. 14 (8 and on: a page that is
    # not there); sequence 1: positions -2 .. 9 of rows 15 .. 26
    cu, length = i32([3, 15, 27]), i32([16, 10])
    P.star_kv_append(c.pages, cu, length, K.to(DEV), K.to(DEV))
    want = torch.zeros((T, 2, D), dtype=F64)
    vals, _ = stored("int8", K)
    there = [3, 4, 5, 6, 25, 26]  # positions 4 .. 7 of sequence 0, 8 and 9 of sequence 1
    want[there] = vals[there]
    for x in P.star_kv_read(c.pages, cu, length, T):
        assert torch.equal(x.cpu().to(F64), want)
    own = [torch.full((T, 2, D), 5.0, dtype=BF16, device=DEV) for _ in range(2)]
    P.star_kv_read(c.pages, cu, length, T, *own)
    want[:3], want[27:] = 5.0, 5.0
    for x in own:
        assert torch.equal(x.cpu().to(F64), want)
    changed = sum(int((a.view(torch.uint8) != b.view(torch.uint8)).any(-1).sum()) for a, b in zip((c.K, c.V), before))
    assert changed <= 2 * 2 * len(there)
    # past the capacity
    P.star_kv_append(c.pages, i32([0, 5, 5]), i32([c.pages.capacity + 40, 0]), K[:5].to(DEV).contiguous(),
                     K[:5].to(DEV).contiguous())
    for x in P.star_kv_read(c.pages, i32([0, 5, 5]), i32([c.pages.capacity + 40, 0]), 5):
        assert not x.any()


# ---- decode ---------------------------------------------------------------------


def run_decode(P, kv, law, q, D, H, Hkv, page, lens, cap, seed=0, types="cyclic", out_dtype=F32, bad_pages=()):
    B = len(lens)
    c = Cache(P, kv, Hkv, D, page, B, cap // page, seed=seed)
    for b, k, v in bad_pages:
        c.table[b, k] = v
    c.dtable.copy_(c.table)
    keys = [rnd((max(n, 0), Hkv, D), 100 * seed + b) for b, n in enumerate(lens)]
    values = [rnd((max(n, 0), Hkv, D), 100 * seed + 50 + b, 0.5) for b, n in enumerate(lens)]
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + max(n, 0))
    if cu[-1]:
        P.star_kv_append(c.pages, i32(cu), i32([max(n, 0) for n in lens]), torch.cat(keys).to(DEV), torch.cat(values).to(DEV))
    pos_type = ref.cyclic(cap, q)
    if types == "random":
        pos_type = torch.randint(0, q, (cap,), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    elif types == "some_bad":
        pos_type[::3] = -1
        pos_type[1::7] = q
        for b, n in enumerate(lens[:-1]):  # the last sequence's query keeps its type, whatever it is
            if n > 0:
                pos_type[n - 1] = (n - 1) % q
    Q = rnd((B, H, D), 7 + seed)
    shape = P.AttnShape(B, cap, H, Hkv, D, q, law)
    O = P.star_attn_decode_paged(shape, c.pages, pos_type.to(DEV), i32(lens), Q.to(DEV), out_dtype=out_dtype)
    k64, v64 = [stored(kv, x)[0] for x in keys], [stored(kv, x)[0] for x in values]
    for b, n in enumerate(lens):
        for u in range(max(n, 0)):
            if not 0 <= int(c.table[b, u // page]) < c.n:
                v64[b][u] = torch.nan
    rO, mag = ref.decode(law, q, pos_type, lens, Q, k64, v64)
    assert ref.off(O, rO, (ref.HALF + ref.SLACK) * mag, out_dtype == BF16) <= 1
    return O, rO


DECODE = [
    # (kv, law, q, D, H, Hkv, page, lengths, capacity, types)
    ("bf16", "star", 1, 64, 1, 1, 8, [1], 8, "cyclic"),
    ("bf16", "star", 4, 64, 12, 12, 16, [347, 1, 16], 512, "cyclic"),
    ("e4m3", "star", 4, 128, 8, 2, 64, [127, 128, 129, 0, 300], 320, "cyclic"),
    ("int8", "dense", 1, 128, 4, 1, 32, [1000, 31, 33], 1024, "cyclic"),
    ("bf16", "dense", 1, 128, 32, 2, 128, [260, 5], 384, "cyclic"),        # 16 heads of one key head
    ("e4m3", "dense", 2, 64, 24, 1, 8, [65, 200], 256, "random"),          # 24: two slices
    ("int8", "tensor2", 4, 64, 6, 3, 256, [255, 256, 257], 512, "random"),
    ("bf16", "star", 8, 64, 2, 2, 16, [190], 256, "random"),               # groups of 8 features
    ("e4m3", "star", 16, 128, 2, 1, 16, [77, 200], 208, "random"),
    ("int8", "star", 2, 64, 4, 4, 1024, [1023], 1024, "cyclic"),
    ("bf16", "star", 4, 64, 4, 2, 32, [90, 64, 150, 33], 160, "some_bad"),
    ("int8", "star", 4, 128, 4, 2, 8, [90, 64, 150, 34], 160, "some_bad"),
]


@pytest.mark.parametrize("case", DECODE, ids=lambda c: "-".join(str(v) for v in c).replace(" ", ""))
def test_decode(P, case):
    kv, law, q, D, H, Hkv, page, lens, cap, types = case
    run_decode(P, kv, law, q, D, H, Hkv, page, lens, cap, types=types)


def test_decode_bf16_results_and_odd_lengths(P):
    O, _ = run_decode(P, "bf16", "star", 4, 64, 4, 2, 16, [0, -3, 40, 17], 64, out_dtype=BF16)
    assert not O[0].any() and not O[1].any()
    # a length past the capacity counts as the capacity
    c = Cache(P, "bf16", 2, 64, 16, 1, 4)
    K = rnd((64, 2, 64), 3).to(DEV)
    P.star_kv_append(c.pages, i32([0, 64]), i32([64]), K, K)
    shape, Q, t = P.AttnShape(1, 64, 4, 2, 64, 4), rnd((1, 4, 64), 4).to(DEV), ref.cyclic(64, 4).to(DEV)
    a, b = (P.star_attn_decode_paged(shape, c.pages, t, i32([n]), Q) for n in (64, 1000))
    assert torch.equal(a, b)


def test_decode_pages_that_are_not_there(P):
    run_decode(P, "e4m3", "star", 4, 64, 4, 2, 16, [100, 70], 112,
               bad_pages=[(0, 2, -1), (0, 6, 1 << 30), (1, 0, 10 ** 6)])


def test_decode_query_of_no_type(P):
    c = Cache(P, "bf16", 1, 64, 8, 2, 2)
    K = rnd((20, 1, 64), 1).to(DEV)
    P.star_kv_append(c.pages, i32([0, 10, 20]), i32([10, 10]), K, K)
    t = ref.cyclic(16, 2)
    t[9] = 2
    O = P.star_attn_decode_paged(P.AttnShape(2, 16, 2, 1, 64, 2), c.pages, t.to(DEV), i32([10, 9]), rnd((2, 2, 64), 2).to(DEV))
    assert not O[0].any() and O[1].any()


def test_decode_many_sequences_and_many_pieces(P):
    """More sequences than threads of a workgroup; and one long sequence,
    whose pieces are joined by many rows of threads."""
    lens = [(37 * b) % 90 for b in range(300)]
    run_decode(P, "int8", "star", 2, 64, 2, 1, 16, lens, 96)
    run_decode(P, "bf16", "star", 2, 64, 2, 1, 64, [20001], 20032, seed=2)


def test_values_that_are_masked_may_be_anything(P):
    """NaN behind a sequence's end, in positions of no type and in feature
    groups that no pair selects does not reach the output."""
    c = Cache(P, "bf16", 1, 64, 8, 1, 8)
    K, V = rnd((40, 1, 64), 1), rnd((40, 1, 64), 2)
    t = ref.cyclic(64, 4)
    t[5] = 9
    want = None
    for poison in (False, True):
        Kp, Vp = K.clone(), V.clone()
        if poison:
            Kp[5], Vp[5] = torch.nan, torch.inf
            # the query's type is 2: keys of type 0 keep groups 0 and 2
            Kp[0:33:4, 0, 16:32] = torch.nan
            c.K[:], c.V[:] = torch.nan, torch.nan
        P.star_kv_append(c.pages, i32([0, 40]), i32([40]), Kp.to(DEV), Vp.to(DEV))
        O = P.star_attn_decode_paged(P.AttnShape(1, 64, 2, 1, 64, 4), c.pages, t.to(DEV), i32([35]), rnd((1, 2, 64), 3).to(DEV))
        want = O if want is None else want
        assert torch.equal(O, want) and bool(torch.isfinite(O).all())


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_scales_of_masked_rows_may_be_anything(P, kv):
    """Rows that are not finite, and places that hold no row, with scale byte
    255: a position of no type, positions behind the end of the sequence."""
    c = Cache(P, kv, 1, 64, 16, 1, 4)
    K, V = rnd((40, 1, 64), 1), rnd((40, 1, 64), 2)
    t = ref.cyclic(64, 4)
    t[5] = 9
    out = []
    for poison in (False, True):
        Kp, Vp = K.clone(), V.clone()
        if poison:
            Kp[5], Vp[5] = torch.nan, torch.inf
            c.ks.fill_(255)
            c.vs.fill_(255)
        P.star_kv_append(c.pages, i32([0, 40]), i32([40]), Kp.to(DEV), Vp.to(DEV))
        out.append(P.star_attn_decode_paged(P.AttnShape(1, 64, 2, 1, 64, 4), c.pages, t.to(DEV), i32([35]), rnd((1, 2, 64), 3).to(DEV)))
    assert torch.equal(out[0], out[1]) and bool(torch.isfinite(out[0]).all())
    # a row that counts and is not finite: NaN for the heads that see it
    t[5] = 1
    assert bool(torch.isnan(P.star_attn_decode_paged(P.AttnShape(1, 64, 2, 1, 64, 4), c.pages, t.to(DEV), i32([35]),
                                                     rnd((1, 2, 64), 3).to(DEV))).all())


def test_offsets_past_32_bits(P):
    """A cache of more than 2^32 bytes whose last pages are used."""
    D, page, Hkv = 128, 1024, 8
    n = (1 << 32) // (page * Hkv * D) + 2
    K, V = (torch.empty((n, Hkv, page, D), dtype=torch.uint8, device=DEV).view(torch.int8) for _ in range(2))
    ks, vs = (torch.zeros((n, Hkv, page), dtype=torch.uint8, device=DEV) for _ in range(2))
    pages = P.KVPages(K, V, i32([[n - 1, 0, n - 2]]), ks, vs)
    T = 2100
    Kn, Vn = rnd((T, Hkv, D), 1), rnd((T, Hkv, D), 2, 0.5)
    P.star_kv_append(pages, i32([0, T]), i32([T]), Kn.to(DEV), Vn.to(DEV))
    got = P.star_kv_read(pages, i32([0, T]), i32([T]), T)
    k64, v64 = stored("int8", Kn)[0], stored("int8", Vn)[0]
    assert torch.equal(got[0].cpu().to(F64), k64) and torch.equal(got[1].cpu().to(F64), v64)
    t, Q = ref.cyclic(3 * page, 2), rnd((1, 8, D), 3)
    O = P.star_attn_decode_paged(P.AttnShape(1, 3 * page, 8, 8, D, 2), pages, t.to(DEV), i32([T]), Q.to(DEV), out_dtype=F32)
    rO, mag = ref.decode("star", 2, t, [T], Q, [k64], [v64])
    assert ref.off(O, rO, (ref.HALF + ref.SLACK) * mag, False) <= 1


def test_matches_the_contiguous_decode(P):
    """The same keys in pages and in a contiguous bf16 cache: both kernels
    against the same 64-bit result."""
    B, S, H, Hkv, D, q = 3, 192, 4, 2, 64, 4
    K, V, Q = rnd((B, S, Hkv, D), 1), rnd((B, S, Hkv, D), 2), rnd((B, H, D), 3)
    lens, t = [192, 1, 77], ref.cyclic(S, q)
    c = Cache(P, "bf16", Hkv, D, 16, B, S // 16)
    P.star_kv_append(c.pages, i32([0, S, 2 * S, 3 * S]), i32([S] * B), K.view(B * S, Hkv, D).to(DEV), V.view(B * S, Hkv, D).to(DEV))
    shape = P.AttnShape(B, S, H, Hkv, D, q)
    a = P.star_attn_decode_paged(shape, c.pages, t.to(DEV), i32(lens), Q.to(DEV), out_dtype=F32)
    b = P.star_attn_decode(shape, t.to(DEV), i32(lens), Q.to(DEV), K.to(DEV), V.to(DEV), out_dtype=F32)
    rO, mag = ref.decode("star", q, t, lens, Q, list(K.double()), list(V.double()))
    for x in (a, b):
        assert ref.off(x, rO, (ref.HALF + ref.SLACK) * mag, False) <= 1


def test_prompts_then_steps_in_a_graph(P):
    """As a server uses them: prompts through the packed forward, their keys
    and values into the cache, then steps of append and decode replayed from
    one graph, each against the packed forward over the sequence so far."""
    H, Hkv, D, q, page, cap = 4, 2, 64, 4, 16, 96
    lens, steps = [33, 1, 60], 6
    B, T = len(lens), sum(lens)
    types = ref.cyclic(cap, q)
    full = {k: rnd((B, cap, h, D), 20 + n) for n, (k, h) in enumerate((("Q", H), ("K", Hkv), ("V", Hkv)))}
    pick = lambda k, ls: torch.cat([full[k][b, :n] for b, n in enumerate(ls)]).to(DEV)
    c = Cache(P, "bf16", Hkv, D, page, B, cap // page)

    def packed(ls):
        cu = [0]
        for n in ls:
            cu.append(cu[-1] + n)
        pack = P.star_attn_pack(q, torch.cat([types[:n] for n in ls]).to(DEV), i32(cu))
        O = P.star_attn_packed_fwd(P.AttnShape(B, cu[-1], H, Hkv, D, q), pack, pick("Q", ls), pick("K", ls), pick("V", ls),
                                   out_dtype=F32)
        return O, cu

    _, cu = packed(lens)
    P.star_kv_append(c.pages, i32(cu), i32(lens), pick("K", lens), pick("V", lens))
    length, one = i32(lens), i32(range(B + 1))
    Q, K, V = (torch.zeros((B, h, D), dtype=BF16, device=DEV) for h in (H, Hkv, Hkv))
    shape, dt = P.AttnShape(B, cap, H, Hkv, D, q), types.to(DEV)
    ws = torch.empty(P.star_attn_decode_paged_workspace_bytes(shape), dtype=torch.uint8, device=DEV)

    def step():
        length.add_(1)
        P.star_kv_append(c.pages, one, length, K, V)
        return P.star_attn_decode_paged(shape, c.pages, dt, length, Q, out_dtype=F32, ws=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):  # (writes zeros at the next position, which the first replay overwrites)
        step()
    s.synchronize()
    length.sub_(1)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = step()
    ls = list(lens)
    for _ in range(steps):
        for x, k in ((Q, "Q"), (K, "K"), (V, "V")):
            x.copy_(torch.stack([full[k][b, n] for b, n in enumerate(ls)]))
        g.replay()
        torch.cuda.synchronize()
        ls = [n + 1 for n in ls]
        assert length.tolist() == ls
        O, cu = packed(ls)
        last = torch.stack([O[z - 1] for z in cu[1:]])
        # each is within its bar of the true result
        _, _, mag = ref.forward("star", q, torch.cat([types[:n] for n in ls]), cu, *(pick(k, ls).cpu() for k in ("Q", "K", "V")))
        bar = 2 * (ref.HALF + ref.SLACK) * torch.stack([mag[z - 1] for z in cu[1:]])
        assert ref.off(out, last.cpu(), bar, False) <= 1


@pytest.mark.parametrize("cap", [64, 4096])  # a workgroup a pair, and shares that are joined
@pytest.mark.parametrize("kv", ["bf16", "int8"])
def test_a_query_that_is_no_number(P, kv, cap):
    D, H, Hkv, page, lens = 64, 4, 2, 16, [50, 64, 1] if cap == 64 else [50, 3000, 1]
    c = Cache(P, kv, Hkv, D, page, 3, cap // page)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    P.star_kv_append(c.pages, i32(cu), i32(lens), rnd((cu[-1], Hkv, D), 1).to(DEV), rnd((cu[-1], Hkv, D), 2).to(DEV))
    Q, t, shape = rnd((3, H, D), 3), ref.cyclic(cap, 4).to(DEV), P.AttnShape(3, cap, H, Hkv, D, 4)
    O = P.star_attn_decode_paged(shape, c.pages, t, i32(lens), Q.to(DEV))
    for b in range(3):
        Qb = Q.clone()
        Qb[b, 1] = torch.nan
        Ob = P.star_attn_decode_paged(shape, c.pages, t, i32(lens), Qb.to(DEV))
        odd = torch.zeros((3, H), dtype=torch.bool, device=DEV)
        odd[b, 1] = True
        assert bool(torch.isnan(Ob[odd]).all()) and torch.equal(Ob[~odd], O[~odd])


def test_two_streams_read_one_cache(P):
    """Decode steps on two streams at once over the same pages."""
    D, H, Hkv, page, lens, cap = 128, 8, 2, 16, [3000, 40, 900], 4096
    c = Cache(P, "e4m3", Hkv, D, page, 3, cap // page)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    P.star_kv_append(c.pages, i32(cu), i32(lens), rnd((cu[-1], Hkv, D), 1).to(DEV), rnd((cu[-1], Hkv, D), 2).to(DEV))
    t, length = ref.cyclic(cap, 4).to(DEV), i32(lens)
    shape = P.AttnShape(3, cap, H, Hkv, D, 4)
    Q = [rnd((3, H, D), 5 + k).to(DEV) for k in range(2)]
    want = [P.star_attn_decode_paged(shape, c.pages, t, length, q) for q in Q]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(6):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k].append(P.star_attn_decode_paged(shape, c.pages, t, length, Q[k]))
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(g, want[k]) for g in got[k])
