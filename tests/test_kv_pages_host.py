"""KVPages on the host: the addresses that the calls take are those of the
tensors that it holds."""

import ctypes

import pytest
import torch


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_tensors_cannot_be_swapped_under_the_pointers(dtype):
    """A page table assigned later would leave the calls with the address of
    the one it replaces, whose memory may be another tensor's by then."""
    import paper_2609_32814_amd as P

    pages = [torch.zeros((3, 2, 8, 64), dtype=dtype) for _ in range(2)]
    scales = [torch.ones((3, 2, 8), dtype=torch.uint8) for _ in range(2)] if dtype == torch.int8 else [None, None]
    table = torch.zeros((2, 4), dtype=torch.int32)
    kv = P.KVPages(*pages, table, *scales)
    for name in ("K_pages", "V_pages", "page_table", "K_scale", "V_scale", "batch", "page_size", "anything"):
        with pytest.raises(AttributeError):
            setattr(kv, name, torch.zeros((2, 4), dtype=torch.int32))
    held = (kv.K_pages, kv.V_pages, kv.page_table, kv.K_scale, kv.V_scale)
    for t, field in zip(held, ("K", "V", "page_table", "K_scale", "V_scale")):
        got = getattr(ctypes.cast(kv.ref, ctypes.POINTER(type(kv._c)))[0], field)
        assert (got or None) == (t.data_ptr() if t is not None else None)
    table[0, 0] = 2  # in place: seen, the same memory
    assert kv.page_table[0, 0] == 2
