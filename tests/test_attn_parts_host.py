"""The gradient of packed attention deals the query heads of a key/value head
out where that shortens its walks by more than the launch that adds the sums
takes: seen from the workspace, which holds the sums."""

import pytest


@pytest.mark.parametrize("n,T,H,Hkv,D,q,law,dealt", [
    (3, 20, 8, 4, 64, 1, "dense", 1),
    (3, 400, 8, 4, 64, 1, "dense", 1),
    (3, 800, 8, 4, 64, 1, "dense", 2),
    (3, 400, 8, 4, 128, 1, "dense", 1),
    (3, 50, 32, 8, 128, 1, "dense", 1),
    (3, 200, 32, 8, 128, 1, "dense", 4),
    (3, 50, 8, 1, 64, 1, "dense", 1),
    (3, 100, 8, 1, 64, 1, "dense", 8),
    (3, 20, 12, 2, 64, 4, "star", 2),
    (1, 4, 2, 1, 64, 1, "dense", 1),
    (0, 30, 2, 1, 64, 1, "dense", 1),     # no sequence
    (48, 800, 8, 4, 64, 1, "dense", 1),   # short ones
    (3, 30, 4, 4, 64, 1, "dense", 1),     # nothing to deal
    (6, 8192, 32, 8, 128, 2, "star", 1),  # items enough
])
def test_where_heads_are_dealt_out(n, T, H, Hkv, D, q, law, dealt):
    import paper_2609_32814_amd as P

    up = lambda b: -(-b // 256) * 256
    # two numbers of every row and head; dK and dV of every part in fp32
    want = up(2 * 4 * H * T) + (up(2 * dealt * 4 * T * Hkv * D) if dealt > 1 else 0)
    assert P.star_attn_packed_bwd_workspace_bytes(P.AttnShape(n, T, H, Hkv, D, q, law)) == want
