"""The paged decode step where the keys of all sequences are dealt out over
the chip (capacities above 2048 positions) and a second launch joins them:
against the plain 64-bit form, every type and law, as the one-launch form in
test_gpu_paged."""

import pytest
import torch

import attn_ref as ref
from test_gpu_paged import BF16, DECODE, DEV, F32, F64, Cache, P, i32, rnd, run_decode, stored  # noqa: F401 (P: fixture)

pytestmark = pytest.mark.gpu

CAP = 4096


@pytest.mark.parametrize("case", DECODE, ids=lambda c: "-".join(str(v) for v in c).replace(" ", ""))
def test_decode(P, case):
    kv, law, q, D, H, Hkv, page, lens, _, types = case
    run_decode(P, kv, law, q, D, H, Hkv, page, lens, CAP, types=types)


@pytest.mark.parametrize("kv,law,q,D,H,Hkv,page", [
    ("e4m3", "dense", 1, 128, 40, 2, 64),      # 20 heads of a key head: a slice of 16 and one of 4
    ("int8", "tensor2", 4, 64, 12, 3, 16),
    ("bf16", "star", 8, 128, 17, 1, 32),
    ("e4m3", "tensor2", 2, 64, 2, 2, 128),
])
def test_ragged_batch_with_empty_sequences(P, kv, law, q, D, H, Hkv, page):
    """Empty sequences first, last and between others, lengths at the borders
    of tiles."""
    run_decode(P, kv, law, q, D, H, Hkv, page, [0, 1, 0, 0, 2500, 32, 0, 33, 4096, 31, 64, 0], CAP, types="random", seed=4)


@pytest.mark.parametrize("kv,law,q,D,H,Hkv", [
    ("e4m3", "star", 4, 128, 8, 2),
    ("int8", "dense", 1, 64, 4, 2),
    ("bf16", "tensor2", 4, 64, 3, 3),
    ("bf16", "star", 2, 128, 4, 2),
])
def test_many_pairs(P, kv, law, q, D, H, Hkv):
    """More than 64 sequences and 128 pairs of a sequence and a key/value head
    (which the join's narrow form takes), some split over many wavefronts and
    some not at all, empty ones inside."""
    lens = [(211 * b) % 97 for b in range(90)]
    for b, n in ((3, 2100), (40, 1000), (64, 3333), (89, 700)):
        lens[b] = n
    lens[10:14] = [0, 0, 0, 0]
    assert len(lens) * Hkv > 128
    run_decode(P, kv, law, q, D, H, Hkv, 16, lens, CAP, seed=6)


def test_more_sequences_than_threads(P):
    run_decode(P, "int8", "star", 2, 64, 2, 1, 16, [(37 * b) % 90 for b in range(300)], 2064)


def test_bf16_results_and_lengths_out_of_range(P):
    O, _ = run_decode(P, "bf16", "star", 4, 64, 4, 2, 16, [0, -3, 40, 2100], CAP, out_dtype=BF16)
    assert not O[0].any() and not O[1].any()
    c = Cache(P, "bf16", 2, 64, 16, 1, CAP // 16)
    K = rnd((CAP, 2, 64), 3).to(DEV)
    P.star_kv_append(c.pages, i32([0, CAP]), i32([CAP]), K, K)
    shape, Q, t = P.AttnShape(1, CAP, 4, 2, 64, 4), rnd((1, 4, 64), 4).to(DEV), ref.cyclic(CAP, 4).to(DEV)
    a, b = (P.star_attn_decode_paged(shape, c.pages, t, i32([n]), Q) for n in (CAP, 1 << 30))
    assert torch.equal(a, b)


@pytest.mark.parametrize("kv", ["bf16", "e4m3", "int8"])
def test_pages_that_are_not_there(P, kv):
    run_decode(P, kv, "star", 4, 64, 4, 2, 16, [2100, 70, 16], CAP,
               bad_pages=[(0, 2, -1), (0, 131, 1 << 30), (0, 64, -2 ** 31), (1, 0, 10 ** 6)])
    # a sequence none of whose pages is there
    O, _ = run_decode(P, kv, "dense", 1, 128, 4, 2, 1024, [3000, 900], CAP, bad_pages=[(0, k, -1) for k in range(3)])
    assert not O[0].any() and O[1].any()


def test_matches_the_one_launch_form(P):
    """The same cache under a table of few pages and one of many: both within
    their bars of one 64-bit result."""
    B, H, Hkv, D, page, q, lens = 3, 6, 2, 64, 32, 4, [1500, 3, 700]
    K = [rnd((n, Hkv, D), 10 + b) for b, n in enumerate(lens)]
    V = [rnd((n, Hkv, D), 20 + b) for b, n in enumerate(lens)]
    Q, cu = rnd((B, H, D), 30), [0]
    for n in lens:
        cu.append(cu[-1] + n)
    rO, mag = ref.decode("star", q, ref.cyclic(1536, q), lens, Q, [x.to(F64) for x in K], [x.to(F64) for x in V])
    for cap in (1536, CAP):
        c = Cache(P, "bf16", Hkv, D, page, B, cap // page)
        P.star_kv_append(c.pages, i32(cu), i32(lens), torch.cat(K).to(DEV), torch.cat(V).to(DEV))
        O = P.star_attn_decode_paged(P.AttnShape(B, cap, H, Hkv, D, q), c.pages, ref.cyclic(cap, q).to(DEV), i32(lens),
                                     Q.to(DEV), out_dtype=F32)
        assert ref.off(O, rO, (ref.HALF + ref.SLACK) * mag, False) <= 1


def test_graph_replays(P):
    """Both launches in a graph, replayed over other lengths, against eager calls."""
    B, H, Hkv, D, page, q = 5, 8, 2, 128, 64, 4
    c = Cache(P, "e4m3", Hkv, D, page, B, CAP // page)
    full = [3000, 700, 4096, 64, 1000]
    cu = [0]
    for n in full:
        cu.append(cu[-1] + n)
    P.star_kv_append(c.pages, i32(cu), i32(full), rnd((cu[-1], Hkv, D), 1).to(DEV), rnd((cu[-1], Hkv, D), 2).to(DEV))
    shape, t, Q, length = P.AttnShape(B, CAP, H, Hkv, D, q), ref.cyclic(CAP, q).to(DEV), rnd((B, H, D), 3).to(DEV), i32(full)
    ws = torch.empty(P.star_attn_decode_paged_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        P.star_attn_decode_paged(shape, c.pages, t, length, Q, ws=ws)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = P.star_attn_decode_paged(shape, c.pages, t, length, Q, ws=ws)
    for lens in (full, [1, 0, 2049, 33, 999], [0, 0, 0, 0, 0], [2999, 700, 4000, 0, 1], full):
        length.copy_(i32(lens))
        ws.fill_(0xff)  # what is left in it is not read
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, P.star_attn_decode_paged(shape, c.pages, t, length, Q))
