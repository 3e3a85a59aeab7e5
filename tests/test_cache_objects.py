"""What the Python calls on the caches take as a cache, and what may be set on it (no GPU needed)."""
import ctypes as C

import pytest

from paper_2310_09443_b200 import binding


def made(kind, **fields):
    """An object of the class as its constructor leaves it (which wants a device)."""
    c = kind.__new__(kind)
    for k, v in dict(dict.fromkeys(kind._FIXED), **fields).items():
        object.__setattr__(c, k, v)
    object.__setattr__(c, "ref", C.byref(binding._Cache()))
    return c


@pytest.mark.parametrize("kind", [binding.CacheBuffers, binding.PackedBuffers])
def test_tensors_are_fixed_and_other_attributes_are_not(kind):
    c = made(kind)
    for name in ("k", "v", "page_table", "lengths", "seen", "scores", "positions", "status"):
        with pytest.raises(binding.G10Error):
            setattr(c, name, 1)
    c.note = 1
    assert c.note == 1


def test_scales_belong_to_the_packed_cache():
    c, p = made(binding.CacheBuffers), made(binding.PackedBuffers)
    c.scales = 3                                         # an attribute as any other, and set again
    c.scales = 4
    assert c.scales == 4
    with pytest.raises(binding.G10Error):
        p.scales = 3
