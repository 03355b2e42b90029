"""What the binding takes for an address (tensors, integers and None, nothing else) and for a type."""

import pytest

from paper_2607_24331_gb300 import dck

A = 1 << 20  # an aligned address that nothing reads


@pytest.mark.parametrize("bad", [b"rows", "rows", bytearray(8), 1.0, [A], object()], ids=lambda b: type(b).__name__)
def test_no_other_object_is_passed_on_as_an_address(bad):
    cache = dck.PagedCache(8, 2, 64, 16, 10, "bf16")
    with pytest.raises(AttributeError):
        dck.dck_paged_append(cache, None, None, 0, bad, 128, A, 128, 0, None, A, None, A, A, stream=0)
    with pytest.raises(AttributeError):
        dck.dck_rope(dck.Rope(64, 1e4), A, 0, 1, 64, 0, 64, 64, A, bad, 64, 64, stream=0)


def test_tensors_integers_and_none():
    import torch
    t = torch.zeros(3)
    assert dck._ptr(t) == t.data_ptr() and dck._ptr(A) == A and dck._ptr(None) is None


@pytest.mark.parametrize("name", ["float32", "fp32", "f16", "torch.bfloat16", "", None])
def test_a_cache_of_another_type_is_refused(name):
    """Anything but f32 was taken for bf16."""
    with pytest.raises(ValueError):
        dck.PagedCache(8, 2, 64, 16, 10, name)
