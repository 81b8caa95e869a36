"""Attention over packed sequences with its gradient, and the paged key-value
cache with the decode step that reads it: the cases they are measured by.

``run`` makes the calls of the public binding where ``own`` is true and
computes the same with elementary torch operations in 32 bits where it is
false.  ``exact`` has the results in 64 bits from the definitions.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
BF16, F32, F64, I32, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8
PAGES = {"bf16": BF16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
# largest magnitude of an 8-bit value, and the power of two below it
TOP = {"e4m3": 448.0, "int8": 127.0}


# ---- cases -------------------------------------------------------------------


def listed():
    return [
        # Three short prompts that a server takes up together: latency.
        dict(name="prompts_short", kind="fwd", law="star", q=4, H=12, Hkv=12, D=64, T=211, n=3, mix=1, lse=False),
        # Forward of a training step over a pack of documents, 12 heads of 64.
        dict(name="pack_forward_24576", kind="fwd", law="star", q=4, H=12, Hkv=12, D=64, T=24576, n=17, mix=2,
             lse=True),
        # Prompts of a model with grouped heads of 128, one far longer than
        # the others, ordinary scores.
        dict(name="prompts_grouped_9001", kind="fwd", law="dense", q=1, H=32, Hkv=8, D=128, T=9001, n=4, mix=3,
             lse=False),
        # Gradient of a small pack under the tensor-square law.
        dict(name="pack_backward_1500", kind="bwd", law="tensor2", q=4, H=12, Hkv=12, D=64, T=1500, n=5, mix=4),
        # Gradient of the training step's pack.
        dict(name="pack_backward_24576", kind="bwd", law="star", q=4, H=12, Hkv=12, D=64, T=24576, n=17, mix=2),
        # Gradient with grouped heads of 128, whose key and value gradients
        # sum over four query heads.
        dict(name="pack_backward_grouped_8192", kind="bwd", law="star", q=2, H=32, Hkv=8, D=128, T=8192, n=6, mix=5),
        # The keys and values of a decode step's new tokens go into an int8 cache.
        dict(name="cache_append_64_tokens", kind="append", kv="int8", Hkv=12, D=64, page=16, T=64, n=64, mix=0,
             cap=2048),
        # Whole prompts go into an e4m3 cache.
        dict(name="cache_append_prompts_16411", kind="append", kv="e4m3", Hkv=8, D=128, page=64, T=16411, n=9, mix=6,
             cap=8192),
        # Cached sequences are read back, to go on with them elsewhere.
        dict(name="cache_read_40000", kind="read", kv="e4m3", Hkv=8, D=128, page=64, T=40000, n=12, mix=7, cap=16384),
        # One sequence being generated, a short bf16 cache: latency.
        dict(name="decode_paged_one", kind="decode", kv="bf16", law="star", q=4, H=12, Hkv=12, D=64, page=16, T=347,
             n=1, mix=0, cap=2048),
        # A serving batch at ragged depths of an e4m3 cache.
        dict(name="decode_paged_64", kind="decode", kv="e4m3", law="star", q=4, H=32, Hkv=8, D=128, page=64, T=131072,
             n=64, mix=8, cap=16384),
        # Three long sequences in an int8 cache: the length is split.
        dict(name="decode_paged_long", kind="decode", kv="int8", law="dense", q=1, H=32, Hkv=8, D=128, page=128,
             T=250007, n=3, mix=9, cap=196608),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(["fwd", "fwd", "bwd", "bwd", "append", "read", "decode", "decode", "decode"])
    D = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8, 12])
    c = dict(kind=kind, Hkv=Hkv, D=D, mix=rng.randint(0, 1 << 20))
    if kind in ("fwd", "bwd", "decode"):
        law = rng.choice(["star", "star", "dense", "tensor2"])
        c.update(law=law, q=4 if law == "tensor2" else 1 if law == "dense" else rng.choice([2, 4, 8]),
                 H=Hkv * rng.choice([1, 1, 2, 4, 8]))
    if kind in ("fwd", "bwd"):
        c.update(T=_log_int(rng, 1, 24576), n=_log_int(rng, 1, 48))
        if kind == "fwd":
            c["lse"] = rng.random() < 0.5
    else:
        c.update(kv=rng.choice(["bf16", "e4m3", "int8"]), page=rng.choice([8, 16, 32, 64, 128, 256]))
        n = _log_int(rng, 1, 64)
        c.update(n=n, T=_log_int(rng, n, 250000 if kind == "decode" else 40000))
        longest = max(_lens(c))
        c["cap"] = -(-max(longest, _log_int(rng, longest, 2 * longest + 64)) // c["page"]) * c["page"]
    return c


def draw(rng):
    """One more case, no dearer than the dearest listed one of its kind."""
    while True:
        c = _draw(rng)
        w = work(c)
        top = [work(v) for v in listed() if v["kind"] == c["kind"]]
        if w["bytes"] <= max(t["bytes"] for t in top) and w["flops"] <= max(t["flops"] for t in top):
            return c


# ---- what a case stands for ----------------------------------------------------


def _lens(c):
    """The lengths of the case's sequences, T in all: ragged (a few much
    longer than the rest) by `mix`, equal shares for mix 0."""
    n, T = c["n"], c["T"]
    r = random.Random(c["mix"])
    w = [1.0] * n if c["mix"] == 0 else [math.exp(r.gauss(0.0, 0.9)) for _ in range(n)]
    edges, s = [0], 0.0
    for v in w:
        s += v
        edges.append(s)
    cut = [int(round(T * e / s)) for e in edges]
    return [cut[k + 1] - cut[k] for k in range(n)]


def _after(c):
    """Cached positions per sequence once the case's tokens are in: the
    prompts themselves, or for one new token each some depth of the cache."""
    lens = _lens(c)
    if c["kind"] == "append" and c["T"] == c["n"]:
        r = random.Random(c["mix"])
        return [r.randint(1, c["cap"]) for _ in lens]
    return lens


def _kept(law, q, i, j):
    """Feature groups that the score of a type-i query and a type-j key keeps."""
    if law == "dense":
        return list(range(q))
    if law == "tensor2":
        return [a for a in range(q) if ((a ^ i) & (a ^ j)) == 0]
    return sorted({i, j})


def _types(n, c):
    """Position types: cyclic, or for the tensor-square law in intervals."""
    p = torch.arange(n, device=DEV)
    if c["law"] == "tensor2":
        return ((p % 768) * c["q"] // 768).to(I32)
    return (p % c["q"]).to(I32)


class _Draws:
    def __init__(self, seed):
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(int(seed))

    def normal(self, shape, std=1.0):
        return (torch.randn(shape, generator=self.gen, device=DEV, dtype=F32) * std).to(BF16)

    def order(self, n):
        return torch.randperm(n, generator=self.gen, device=DEV)


def _starts(lens):
    cu = [0]
    for v in lens:
        cu.append(cu[-1] + v)
    return cu


def _page_table(c, r):
    """Pages for every sequence, in an order of their own: (table, pages)."""
    per = c["cap"] // c["page"]
    after = _after(c)
    need = [-(-v // c["page"]) for v in after]
    total = sum(need) + 3
    ids = r.order(total).to(I32)
    table = torch.zeros((c["n"], per), dtype=I32, device=DEV)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = ids[at:at + k]
        at += k
    return table, total


def _slots(c, table, first, count):
    """Page and place of `count` positions of sequence b from `first[b]` on,
    for all sequences in turn."""
    pos = torch.cat([torch.arange(f, f + n, device=DEV) for f, n in zip(first, count)])
    seq = torch.repeat_interleave(torch.arange(c["n"], device=DEV), torch.tensor(count, device=DEV))
    return table[seq, pos // c["page"]].long(), pos % c["page"]


def _inputs(c, seed):
    """The tensors of a case, made from the seed alone."""
    r, t = _Draws(seed), {}
    D, Hkv, T = c["D"], c["Hkv"], c["T"]
    lens = _lens(c)
    if c["kind"] in ("fwd", "bwd"):
        t["Q"], t["K"], t["V"] = r.normal((T, c["H"], D)), r.normal((T, Hkv, D)), r.normal((T, Hkv, D))
        if c["kind"] == "bwd":
            t["dO"] = r.normal((T, c["H"], D))
        t["types"] = torch.cat([_types(n, c) for n in lens])
        t["cu"] = torch.tensor(_starts(lens), dtype=I32, device=DEV)
        if c["kind"] == "bwd":  # what the forward of the same step left
            t["O"], t["lse"] = _forward_plain(c, t)
        return t
    t["table"], n_pages = _page_table(c, r)
    t["len"] = torch.tensor(_after(c), dtype=I32, device=DEV)
    shape = (n_pages, Hkv, c["page"], D)
    if c["kind"] == "append":
        t["K"], t["V"] = r.normal((T, Hkv, D)), r.normal((T, Hkv, D), 0.3)
        t["cu"] = torch.tensor(_starts(lens), dtype=I32, device=DEV)
        for name in ("K", "V"):
            t[name + "_pages"] = torch.zeros(shape, dtype=U8 if c["kv"] != "bf16" else BF16, device=DEV)
            t[name + "_scale"] = torch.ones(shape[:3], dtype=U8, device=DEV) if c["kv"] != "bf16" else None
    else:
        for name, std in (("K", 1.0), ("V", 0.3)):
            t[name + "_pages"], t[name + "_scale"] = _to_pages(c["kv"], r.normal(shape, std))
        if c["kind"] == "read":
            t["cu"] = torch.tensor(_starts(lens), dtype=I32, device=DEV)
        else:
            t["Q"] = r.normal((c["n"], c["H"], D))
            t["types"] = _types(c["cap"], c)
    for name in ("K_pages", "V_pages"):
        t[name] = t[name].view(PAGES[c["kv"]])
    return t


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if own:
        _handles(st)
    return st


def _handles(st):
    """Shapes, plan and workspace, which a program keeps over layers and steps."""
    import paper_2609_32814_amd as starq
    c = st["case"]
    st["lib"] = starq
    if c["kind"] in ("fwd", "bwd"):
        st["shape"] = starq.AttnShape(c["n"], c["T"], c["H"], c["Hkv"], c["D"], c["q"], c["law"])
        st["pack"] = starq.star_attn_pack(c["q"], st["types"], st["cu"])
        if c["kind"] == "bwd":
            st["ws"] = _bytes(starq.star_attn_packed_bwd_workspace_bytes(st["shape"]))
        return
    st["pages"] = starq.KVPages(st["K_pages"], st["V_pages"], st["table"], st["K_scale"], st["V_scale"])
    if c["kind"] == "decode":
        st["shape"] = starq.AttnShape(c["n"], c["cap"], c["H"], c["Hkv"], c["D"], c["q"], c["law"])
        st["ws"] = _bytes(starq.star_attn_decode_paged_workspace_bytes(st["shape"]))


def _bytes(n):
    return torch.empty(max(n, 16), dtype=U8, device=DEV)


# ---- one pass ------------------------------------------------------------------


def run(st):
    c = st["case"]
    if not own:
        return _run_plain(c, st)
    if "lib" not in st:
        _handles(st)
    lib, kind = st["lib"], c["kind"]
    if kind == "fwd":
        return lib.star_attn_packed_fwd(st["shape"], st["pack"], st["Q"], st["K"], st["V"], want_lse=c["lse"])
    if kind == "bwd":
        return lib.star_attn_packed_bwd(st["shape"], st["pack"], st["dO"], st["Q"], st["K"], st["V"], st["O"],
                                        st["lse"], ws=st["ws"])
    if kind == "append":
        lib.star_kv_append(st["pages"], st["cu"], st["len"], st["K"], st["V"])
        return lib.star_kv_read(st["pages"], st["cu"], st["len"], c["T"])
    if kind == "read":
        return lib.star_kv_read(st["pages"], st["cu"], st["len"], c["T"])
    return lib.star_attn_decode_paged(st["shape"], st["pages"], st["types"], st["len"], st["Q"], ws=st["ws"])


# ---- the plain forms -------------------------------------------------------------


def _run_plain(c, st):
    if c["kind"] == "fwd":
        O, lse = _forward_plain(c, st)
        return (O, lse) if c["lse"] else O
    if c["kind"] == "bwd":
        return _backward_plain(c, st)
    if c["kind"] == "append":
        count = _lens(c)
        page, place = _slots(c, st["table"], [a - n for a, n in zip(_after(c), count)], count)
        for name in ("K", "V"):
            vals, scale = _to_pages(c["kv"], st[name])
            pages = st[name + "_pages"]
            if scale is None:
                pages[page, :, place] = vals
            else:
                pages.view(U8)[page, :, place] = vals
                st[name + "_scale"][page, :, place] = scale
        return _read_plain(c, st, page, place)
    if c["kind"] == "read":
        return _read_plain(c, st, *_slots(c, st["table"], [0] * c["n"], _lens(c)))
    return _decode_plain(c, st)


def _group_masks(c, tq, tk):
    """(scale [n_q, n_k], one 0/1 mask [n_q, n_k] per feature group)."""
    q, m = c["q"], c["D"] // c["q"]
    keep = torch.zeros((q, q, q), dtype=F32, device=DEV)
    for i in range(q):
        for j in range(q):
            for a in _kept(c["law"], q, i, j):
                keep[a, i, j] = 1.0
    norm = 1.0 / torch.sqrt(keep.sum(0) * m)
    pick = lambda w: w[tq.long()][:, tk.long()]
    return pick(norm), None if c["law"] == "dense" else [pick(keep[a]) for a in range(q)]


def _scores_plain(c, Q, K, scale, masks):
    """Scaled scores [H, n_q, n_k] of Q [H, n_q, D] and K [H, n_k, D]."""
    if masks is None:
        return Q @ K.transpose(1, 2) * scale
    m, s = c["D"] // c["q"], 0.0
    for a, keep in enumerate(masks):
        f = slice(a * m, (a + 1) * m)
        s = s + (Q[:, :, f] @ K[:, :, f].transpose(1, 2)) * keep
    return s * scale


def _sequences(c, st):
    """(first, last, types, causal mask) of each sequence that has tokens."""
    at = 0
    for n in _lens(c):
        if n:
            future = torch.ones((n, n), dtype=torch.bool, device=DEV).triu_(1)
            yield at, at + n, st["types"][at:at + n], future
        at += n


def _heads(x, rep=1):
    """[n, H, D] of any type to [H rep, n, D] in 32 bits."""
    x = x.to(F32).transpose(0, 1)
    return torch.repeat_interleave(x, rep, 0) if rep > 1 else x


def _forward_plain(c, st):
    T, H, rep = c["T"], c["H"], c["H"] // c["Hkv"]
    O = torch.empty((T, H, c["D"]), dtype=BF16, device=DEV)
    lse = torch.empty((H, T), dtype=F32, device=DEV)
    for a, z, types, future in _sequences(c, st):
        s = _scores_plain(c, _heads(st["Q"][a:z]), _heads(st["K"][a:z], rep), *_group_masks(c, types, types))
        s = s.masked_fill(future, float("-inf"))
        top = s.amax(-1, keepdim=True)
        e = torch.exp(s - top)
        total = e.sum(-1, keepdim=True)
        O[a:z] = ((e @ _heads(st["V"][a:z], rep)) / total).transpose(0, 1).to(BF16)
        lse[:, a:z] = (top + torch.log(total))[..., 0]
    return O, lse


def _backward_plain(c, st):
    H, Hkv, D, rep, m = c["H"], c["Hkv"], c["D"], c["H"] // c["Hkv"], c["D"] // c["q"]
    dQ, dK, dV = (torch.empty_like(st[k]) for k in ("Q", "K", "V"))
    for a, z, types, future in _sequences(c, st):
        n = z - a
        Q, dO = _heads(st["Q"][a:z]), _heads(st["dO"][a:z])
        K, V = _heads(st["K"][a:z], rep), _heads(st["V"][a:z], rep)
        scale, masks = _group_masks(c, types, types)
        p = torch.exp(_scores_plain(c, Q, K, scale, masks) - st["lse"][:, a:z, None]).masked_fill(future, 0.0)
        delta = (dO * _heads(st["O"][a:z])).sum(-1, keepdim=True)
        ds = p * (dO @ V.transpose(1, 2) - delta) * scale
        gV = p.transpose(1, 2) @ dO
        if masks is None:
            gQ, gK = ds @ K, ds.transpose(1, 2) @ Q
        else:
            f = [slice(g * m, (g + 1) * m) for g in range(c["q"])]
            gQ = torch.cat([(ds * keep) @ K[:, :, f[g]] for g, keep in enumerate(masks)], -1)
            gK = torch.cat([(ds * keep).transpose(1, 2) @ Q[:, :, f[g]] for g, keep in enumerate(masks)], -1)
        dQ[a:z] = gQ.transpose(0, 1).to(BF16)
        dK[a:z] = gK.view(Hkv, rep, n, D).sum(1).transpose(0, 1).to(BF16)
        dV[a:z] = gV.view(Hkv, rep, n, D).sum(1).transpose(0, 1).to(BF16)
    return dQ, dK, dV


def _pow2(e):
    """2^e in 32 bits for whole e in [-126, 127]."""
    return ((e.to(I32) + 127) << 23).view(F32)


def _to_pages(kv, x):
    """Rows [..., D] as they are cached: (values, scale bytes).  A byte b is
    the scale 2^(b - 127), the smallest at which the row's largest magnitude
    fits the type."""
    if kv == "bf16":
        return x, None
    x = x.to(F32)
    frac, exp = torch.frexp(x.abs().amax(-1, keepdim=True))  # frac in [0.5, 1), amax = frac 2^exp
    ftop, etop = math.frexp(TOP[kv])
    e = (exp - etop + (frac > ftop).to(exp.dtype)).clamp(min=-126)
    y = x * _pow2(-e)
    vals = y.to(torch.float8_e4m3fn).view(U8) if kv == "e4m3" else torch.round(y).to(torch.int8).view(U8)
    return vals, (e + 127).to(U8)[..., 0]


def _values_plain(c, st, name, page, place):
    """Cached rows [n, Hkv, D] in 32 bits."""
    pages = st[name + "_pages"]
    if c["kv"] == "bf16":
        return pages[page, :, place].to(F32)
    rows = pages.view(U8)[page, :, place].view(PAGES[c["kv"]]).to(F32)
    return rows * _pow2(st[name + "_scale"][page, :, place].to(I32)[..., None] - 127)


def _read_plain(c, st, page, place):
    return tuple(_values_plain(c, st, name, page, place).to(BF16) for name in ("K", "V"))


def _decode_plain(c, st):
    rep = c["H"] // c["Hkv"]
    O = torch.empty((c["n"], c["H"], c["D"]), dtype=BF16, device=DEV)
    for b, n in enumerate(_after(c)):
        if n == 0:
            O[b] = 0
            continue
        pos = torch.arange(n, device=DEV)
        page, place = st["table"][b, pos // c["page"]].long(), pos % c["page"]
        K, V = (_heads(_values_plain(c, st, name, page, place), rep) for name in ("K", "V"))
        types = st["types"][:n]
        s = _scores_plain(c, _heads(st["Q"][b:b + 1]), K, *_group_masks(c, types[n - 1:], types))
        e = torch.exp(s - s.amax(-1, keepdim=True))
        O[b] = ((e @ V) / e.sum(-1, keepdim=True))[:, 0].to(BF16)
    return O


# ---- what a pass cannot do without -----------------------------------------------


def _kept_mean(c):
    q = c["q"]
    return sum(len(_kept(c["law"], q, i, j)) for i in range(q) for j in range(q)) / (q * q) * (c["D"] // q)


def work(case):
    c = case
    kind, T, Hkv, D, n = c["kind"], c["T"], c["Hkv"], c["D"], c["n"]
    if kind in ("fwd", "bwd"):
        H, keep = c["H"], _kept_mean(c)
        pairs = H * sum(v * (v + 1) / 2 for v in _lens(c))
        if kind == "fwd":
            return dict(bytes=int(2 * T * D * (2 * H + 2 * Hkv) + 4 * T + (4 * T * H if c["lse"] else 0)),
                        flops=int(pairs * 2 * (keep + D)))
        return dict(bytes=int(2 * T * D * (4 * H + 4 * Hkv) + 4 * T + 4 * T * H),
                    flops=int(pairs * 2 * (3 * keep + 2 * D)))
    elem, scale = (2, 0) if c["kv"] == "bf16" else (1, 1)
    row = D * elem + scale
    if kind in ("append", "read"):
        passes = 2 if kind == "append" else 1  # written, then read back
        return dict(bytes=int(passes * 2 * T * Hkv * (2 * D + row)), flops=int(passes * 2 * T * Hkv * D))
    keys, keep = sum(_after(c)), _kept_mean(c)
    return dict(bytes=int(keys * Hkv * ((keep + D) * elem + 2 * scale) + 4 * n * c["H"] * D + 4 * c["cap"]),
                flops=int(keys * c["H"] * 2 * (keep + D)))


# ---- the same in 64 bits -----------------------------------------------------------


def _attend64(c, Q, K, V, tq, tk, last):
    """(O [n_q, H, D], lse [H, n_q]) type pair by type pair; query r sees the
    keys 0 .. last[r]."""
    rep, m = c["H"] // c["Hkv"], c["D"] // c["q"]
    n_q, n_k = Q.shape[0], K.shape[0]
    seen = torch.arange(n_k, device=DEV)[None, :] <= last[:, None]
    rows = [torch.nonzero(tq == i).flatten() for i in range(c["q"])]
    cols = [torch.nonzero(tk == j).flatten() for j in range(c["q"])]
    Os, lses = [], []
    for h in range(c["H"]):
        Qh, Kh, Vh = Q[:, h], K[:, h // rep], V[:, h // rep]
        parts = []
        for i in range(c["q"]):
            if not rows[i].numel():
                continue
            across = []
            for j in range(c["q"]):
                if not cols[j].numel():
                    continue
                f = torch.cat([torch.arange(a * m, (a + 1) * m, device=DEV) for a in _kept(c["law"], c["q"], i, j)])
                across.append(Qh[rows[i]][:, f] @ Kh[cols[j]][:, f].t().contiguous() / math.sqrt(f.numel()))
            parts.append(torch.cat(across, 1))
        # back from the order by types to the order of positions
        s = torch.cat(parts)[torch.argsort(torch.cat(rows))][:, torch.argsort(torch.cat(cols))]
        s = torch.where(seen, s, torch.full_like(s, float("-inf")))
        Os.append(torch.softmax(s, -1) @ Vh)
        lses.append(torch.logsumexp(s, -1))
    return torch.stack(Os, 1), torch.stack(lses)


def _gradients64(c, t):
    """(dQ, dK, dV) from the output and the log-sum-exp that came in, type
    pair by type pair."""
    rep, m = c["H"] // c["Hkv"], c["D"] // c["q"]
    dQ, dK, dV = (torch.zeros(t[k].shape, dtype=F64, device=DEV) for k in ("Q", "K", "V"))
    at = 0
    for n in _lens(c):
        types = t["types"][at:at + n]
        of = [torch.nonzero(types == i).flatten() + at for i in range(c["q"])]
        at += n
        for i, j in ((i, j) for i in range(c["q"]) for j in range(c["q"])):
            r, u = of[i], of[j]
            if not (r.numel() and u.numel()):
                continue
            f = torch.cat([torch.arange(a * m, (a + 1) * m, device=DEV) for a in _kept(c["law"], c["q"], i, j)])
            norm, seen = 1.0 / math.sqrt(f.numel()), u[None, :] <= r[:, None]
            for h in range(c["H"]):
                g = h // rep
                Qf, Kf = t["Q"][r, h].to(F64)[:, f], t["K"][u, g].to(F64)[:, f]
                up, O, V = t["dO"][r, h].to(F64), t["O"][r, h].to(F64), t["V"][u, g].to(F64)
                s = torch.where(seen, Qf @ Kf.t().contiguous() * norm, float("-inf"))
                p = torch.exp(s - t["lse"][h, r].to(F64)[:, None])
                ds = p * (up @ V.t().contiguous() - (up * O).sum(1)[:, None]) * norm
                dQ[r[:, None], h, f[None, :]] += ds @ Kf
                dK[u[:, None], g, f[None, :]] += ds.t().contiguous() @ Qf
                dV[u, g] += p.t().contiguous() @ up
    return dQ, dK, dV


def _cached64(c, t, name, b, first, count):
    """Cached rows of sequence b, read page by page."""
    out, size = [], c["page"]
    for k in range(first // size, -(-(first + count) // size)):
        lo, hi = max(first, k * size) - k * size, min(first + count, (k + 1) * size) - k * size
        g = int(t["table"][b, k].item())
        rows = t[name + "_pages"][g].to(F32).to(F64)[:, lo:hi]
        if c["kv"] != "bf16":
            rows = rows * _pow64(t[name + "_scale"][g, :, lo:hi].long() - 127)[..., None]
        out.append(rows)
    return torch.cat(out, 1).transpose(0, 1)


def _pow64(e):
    """2^e for whole e in [-1022, 1023]."""
    return ((e + 1023) << 52).view(F64)


def _stored64(kv, x):
    """The values that rows stand for once they are cached."""
    x = x.to(F64)
    if kv == "bf16":
        return x
    top = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -126).long()
    for k in range(-126, 128):  # one up as long as the row does not fit
        e = torch.where(top > TOP[kv] * 2.0 ** k, k + 1, e)
    y = x * _pow64(-e)
    if kv == "int8":
        return torch.round(y) * _pow64(e)
    # e4m3: three bits after the leading one, the smallest exponent -6
    step = _pow64(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).long() - 3)
    return torch.round(y / step) * step * _pow64(e)


def exact(case, seed):
    c, t = case, _inputs(case, seed)
    if c["kind"] == "append":
        return tuple(_stored64(c["kv"], t[name]) for name in ("K", "V"))
    if c["kind"] == "read":
        return tuple(torch.cat([_cached64(c, t, name, b, 0, n) for b, n in enumerate(_lens(c)) if n])
                     for name in ("K", "V"))
    if c["kind"] == "decode":
        O = torch.zeros((c["n"], c["H"], c["D"]), dtype=F64, device=DEV)
        for b, n in enumerate(_after(c)):
            if n:
                K, V = (_cached64(c, t, name, b, 0, n).contiguous() for name in ("K", "V"))
                O[b] = _attend64(c, t["Q"][b:b + 1].to(F64), K, V, t["types"][n - 1:n], t["types"][:n],
                                 torch.tensor([n - 1], device=DEV))[0][0]
        return O
    if c["kind"] == "bwd":
        return _gradients64(c, t)
    parts, at = [], 0
    for n in _lens(c):
        if n:
            types = t["types"][at:at + n]
            parts.append(_attend64(c, *(t[k][at:at + n].to(F64) for k in ("Q", "K", "V")), types, types,
                                   torch.arange(n, device=DEV)))
        at += n
    O, lse = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts], 1)
    return (O, lse) if c["lse"] else O
