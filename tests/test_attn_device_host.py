"""Attention over packs and paged caches, called with tensors of a device that
is not the current one: the library is entered with theirs current (it asks for
the device's compute units and sets its kernels' LDS limit there)."""

import contextlib
import types

import pytest
import torch

BF16, I32, U8 = torch.bfloat16, torch.int32, torch.uint8


@pytest.fixture(scope="module")
def P():
    import paper_2609_32814_amd as P
    import paper_2609_32814_amd.binding  # noqa: F401
    return P


def test_context(P, monkeypatch):
    on = P.binding._on
    monkeypatch.setattr(P.binding, "_current", lambda: 1)
    assert on(torch.device("cuda", 1)) is on(torch.device("cuda", 1))
    other = on(torch.device("cuda", 0))
    assert isinstance(other, torch.cuda.device) and other.idx == 0


def test_every_call_enters_the_library_on_the_tensors_device(P, monkeypatch):
    """CPU tensors in the place of a device's, a library that notes how it was
    entered."""
    b, seen, depth = P.binding, [], [None]

    @contextlib.contextmanager
    def on(device):
        depth[0] = device
        yield
        depth[0] = None

    def entry(name):
        real = getattr(b.LIB, name)

        def call(*args):
            seen.append((name, depth[0]))
            return real(*args) if name.endswith("_bytes") else 0
        return call

    names = ("star_attn_pack", "star_attn_pack_bytes", "star_attn_packed_fwd", "star_attn_packed_bwd",
             "star_attn_packed_bwd_workspace_bytes", "star_kv_append", "star_kv_read", "star_attn_decode_paged",
             "star_attn_decode_paged_workspace_bytes")
    fake = types.SimpleNamespace(**{n: entry(n) for n in names})
    for name, value in (("LIB", fake), ("_on", on), ("_gpu", lambda device: None), ("_stream", lambda device: 0)):
        monkeypatch.setattr(b, name, value)

    sh, T = P.AttnShape(1, 8, 2, 1, 64, 2), 8
    Q, K, cu = torch.zeros((T, 2, 64), dtype=BF16), torch.zeros((T, 1, 64), dtype=BF16), torch.tensor([0, T], dtype=I32)
    t, lse, length = torch.zeros(T, dtype=I32), torch.zeros((2, T)), torch.tensor([T], dtype=I32)
    pack = b.star_attn_pack(2, t, cu)
    b.star_attn_packed_fwd(sh, pack, Q, K, K)
    b.star_attn_packed_bwd(sh, pack, Q, Q, K, K, Q, lse)
    kv = P.KVPages(torch.zeros((2, 1, 8, 64), dtype=BF16), torch.zeros((2, 1, 8, 64), dtype=BF16), torch.zeros((1, 1), dtype=I32))
    b.star_kv_append(kv, cu, length, K, K)
    b.star_kv_read(kv, cu, length, T)
    b.star_attn_decode_paged(sh, kv, t, length, Q[:1])
    cpu = torch.device("cpu")
    assert {n for n, _ in seen} == set(names)
    # (a plan's size does not depend on the device)
    assert all(d == cpu for n, d in seen if n != "star_attn_pack_bytes"), seen
