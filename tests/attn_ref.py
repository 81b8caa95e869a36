"""Plain 64-bit attention over packs and paged caches, on the CPU, with the
absolute sums that bound a kernel's rounding errors.

Bars.  Products of bf16 operands are exact in fp32.  A probability (or dS)
that enters a product as bf16 is off by at most half a step, HALF = 2^-8 of
itself, so a sum of p v is off by HALF sum p |v|; a bf16 result by HALF of
itself once more.  SLACK = 2^-14 covers what fp32 adds per term: scores of at
most 2^5 summed over 128 products (2^5 2^-23 2^7 / 2 < 2^-12 at worst, 2^-16
with errors of both signs), the hardware's exp2 and rsqrt (2^-22) and sums in
another order.
"""

import math

import torch

HALF, SLACK = 2.0 ** -8, 2.0 ** -14
F64 = torch.float64


def kept(law, q, i, j):
    if law == "dense":
        return list(range(q))
    if law == "tensor2":
        return [a for a in range(q) if ((a ^ i) & (a ^ j)) == 0]
    return sorted({i, j})


def cyclic(n, q):
    return (torch.arange(n) % q).to(torch.int32)


def pair_scores(law, q, Q, K, tq, tk):
    """(scaled scores [n_q, n_k], keep [q, n_q, n_k], scale [n_q, n_k]) of one
    head; pairs with a type out of range get keep = 0, scale = 0."""
    D = Q.shape[1]
    m = D // q
    table = torch.zeros((q + 1, q + 1, q), dtype=F64)
    for i in range(q):
        for j in range(q):
            table[i, j, kept(law, q, i, j)] = 1.0
    clean = lambda t: torch.where((t >= 0) & (t < q), t, torch.full_like(t, q)).long()
    keep = table[clean(tq)][:, clean(tk)].permute(2, 0, 1)
    n = keep.sum(0) * m
    scale = torch.where(n > 0, n.clamp(min=1.0) ** -0.5, torch.zeros_like(n))
    s = sum((Q[:, a * m:(a + 1) * m] @ K[:, a * m:(a + 1) * m].t()) * keep[a] for a in range(q))
    return s * scale, keep, scale


def valid(t, q):
    return (t >= 0) & (t < q)


def forward(law, q, types, cu, Q, K, V):
    """(O, lse, sum p |v|) of a pack; Q [T, H, D] and so on, any float type.
    Rows of no sequence or of a type out of range: zeros, lse -inf."""
    T, H, D = Q.shape
    rep = H // K.shape[1]
    Q, K, V = (x.to(F64) for x in (Q, K, V))
    O, mag = torch.zeros((T, H, D), dtype=F64), torch.zeros((T, H, D), dtype=F64)
    lse = torch.full((H, T), -math.inf, dtype=F64)
    for a, z in zip(cu[:-1], cu[1:]):
        t = types[a:z]
        rows = torch.nonzero(valid(t, q)).flatten()
        if not rows.numel():
            continue
        t, r = t[rows], rows + a
        see = rows[None, :] <= rows[:, None]
        for h in range(H):
            s, _, _ = pair_scores(law, q, Q[r, h], K[r, h // rep], t, t)
            s = s.masked_fill(~see, -math.inf)
            p = torch.softmax(s, -1)
            O[r, h] = p @ V[r, h // rep]
            mag[r, h] = p @ V[r, h // rep].abs()
            lse[h, r] = torch.logsumexp(s, -1)
    return O, lse, mag


def backward(law, q, types, cu, dO, Q, K, V, O, lse):
    """((dQ, dK, dV), (bars)): the gradients from O and lse as given, and what
    a kernel's may be off by before its output is rounded."""
    T, H, D = Q.shape
    Hkv = K.shape[1]
    rep, m = H // Hkv, D // q
    dO, Q, K, V, O, lse = (x.to(F64) for x in (dO, Q, K, V, O, lse))
    g = [torch.zeros_like(Q), torch.zeros_like(K), torch.zeros_like(V)]
    bar = [torch.zeros_like(x) for x in g]
    for a, z in zip(cu[:-1], cu[1:]):
        t = types[a:z]
        rows = torch.nonzero(valid(t, q)).flatten()
        if not rows.numel():
            continue
        t, r = t[rows], rows + a
        see = rows[None, :] <= rows[:, None]
        for h in range(H):
            k = h // rep
            s, keep, scale = pair_scores(law, q, Q[r, h], K[r, k], t, t)
            p = torch.exp(s - lse[h, r][:, None]).masked_fill(~see, 0.0)
            delta = (dO[r, h] * O[r, h]).sum(1)[:, None]
            ds = p * (dO[r, h] @ V[r, k].t() - delta) * scale
            # dP and delta as fp32 sums: their own terms bound them
            size = dO[r, h].abs() @ V[r, k].abs().t() + (dO[r, h] * O[r, h]).abs().sum(1)[:, None]
            err = HALF * ds.abs() + SLACK * p * size * scale
            g[2][r, k] += p.t() @ dO[r, h]
            bar[2][r, k] += (HALF + SLACK) * (p.t() @ dO[r, h].abs())
            for c in range(q):
                f = slice(c * m, (c + 1) * m)
                g[0][r, h, f] += (ds * keep[c]) @ K[r, k, f]
                bar[0][r, h, f] += (err * keep[c]) @ K[r, k, f].abs()
                g[1][r, k, f] += (ds * keep[c]).t() @ Q[r, h, f]
                bar[1][r, k, f] += (err * keep[c]).t() @ Q[r, h, f].abs()
    return g, bar


def decode(law, q, pos_type, lens, Q, keys, values):
    """(O, sum p |v|) of one new token per sequence; keys[b], values[b]
    [len_b, Hkv, D] (rows of NaN: positions that are not there)."""
    B, H, D = Q.shape
    Q = Q.to(F64)
    O, mag = torch.zeros((B, H, D), dtype=F64), torch.zeros((B, H, D), dtype=F64)
    for b in range(B):
        n = lens[b]
        if n <= 0 or not valid(pos_type[n - 1], q):
            continue
        there = ~torch.isnan(values[b][:n, 0, 0])
        u = torch.nonzero(valid(pos_type[:n], q) & there).flatten()
        if not u.numel():
            continue
        for h in range(H):
            k = h // (H // keys[b].shape[1])
            s, _, _ = pair_scores(law, q, Q[b, h][None], keys[b][u, k], pos_type[n - 1:n], pos_type[u])
            p = torch.softmax(s, -1)
            O[b, h], mag[b, h] = (p @ values[b][u, k])[0], (p @ values[b][u, k].abs())[0]
    return O, mag


def off(got, ref, bar, rounded):
    """Largest error over its bar (at most 1 for a right kernel); `rounded`:
    the result is bf16.  Equal where the bar is zero."""
    got, ref = got.detach().to(F64).cpu(), ref.to(F64)
    lim = bar + (HALF * (ref.abs() + bar) if rounded else 0.0) + 1e-30
    assert bool(torch.isfinite(got).all())
    return float(((got - ref).abs() / lim).max()) if got.numel() else 0.0
