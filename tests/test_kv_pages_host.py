"""The paged cache on the host: KVPages keeps the tensors whose addresses the
calls take; the sizes that a launch can hold."""

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


def test_rows_that_no_launch_holds_are_refused():
    """2^28 rows and more would take 2^32 threads (fake pointers, never read:
    a refusal comes first; one row fewer is refused for a pointer instead)."""
    import paper_2609_32814_amd as P

    b = P.binding
    shape = {v: k for k, v in b.STATUS_NAMES.items()}["STAR_ERR_SHAPE"]
    arg = {v: k for k, v in b.STATUS_NAMES.items()}["STAR_ERR_ARG"]
    V = ctypes.c_void_p
    pg = b._CKvPages(10, 16, 2, 64, 2, 4, 1, 16, 16, 16, 16, 16)
    top = (1 << 28) - 16
    for T in (top + 1, 1 << 28, 0x7fffff00, 1 << 40):
        assert b.LIB.star_kv_append(ctypes.byref(pg), V(16), V(16), T, V(16), V(16), 1, None) == shape
        assert b.LIB.star_kv_read(ctypes.byref(pg), V(16), V(16), T, V(16), V(16), 1, 0, None) == shape
    assert b.LIB.star_kv_append(ctypes.byref(pg), V(16), V(16), top, None, V(16), 1, None) == arg
    assert b.LIB.star_kv_read(ctypes.byref(pg), V(16), V(16), top, None, V(16), 1, 0, None) == arg


def test_no_sequence_at_all():
    """A cache of no sequences has no table and no lengths: appending its
    rows, which are outside every sequence, is done at once."""
    import paper_2609_32814_amd as P

    b, V = P.binding, ctypes.c_void_p
    names = {v: k for k, v in b.STATUS_NAMES.items()}
    none = b._CKvPages(10, 16, 2, 64, 0, 4, 1, 16, 16, 16, 16, None)
    assert b.LIB.star_kv_append(ctypes.byref(none), V(16), None, 5, V(16), V(16), 1, None) == 0
    assert b.LIB.star_kv_append(ctypes.byref(none), None, None, 5, V(16), V(16), 1, None) == names["STAR_ERR_ARG"]
    one = b._CKvPages(10, 16, 2, 64, 1, 4, 1, 16, 16, 16, 16, 16)
    assert b.LIB.star_kv_append(ctypes.byref(one), V(16), None, 5, V(16), V(16), 1, None) == names["STAR_ERR_ARG"]
    one.page_table = None
    assert b.LIB.star_kv_append(ctypes.byref(one), V(16), V(16), 5, V(16), V(16), 1, None) == names["STAR_ERR_ARG"]
