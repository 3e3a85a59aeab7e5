"""What the Python calls on the caches take as a cache, and what may be set on it (no GPU needed)."""
import ctypes as C
from types import SimpleNamespace

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


FAKE = 1 << 20                                          # an address that is aligned; never followed


def described(packed):
    c = binding._Cache(0, 2, 4, 64, 16, 8, 100, FAKE, FAKE, 16 * 4 * 64, 4 * 64, 64, FAKE, 8, FAKE, None, FAKE, None, FAKE)
    return binding._Packed(c, 0, FAKE) if packed else c


def test_anything_with_the_fields_is_a_cache():
    """... but a packed one is not an ordinary one, nor the other way about."""
    own, theirs = SimpleNamespace(ref=C.byref(described(False))), made(binding.PackedBuffers)
    object.__setattr__(theirs, "ref", C.byref(described(True)))
    assert binding.g10_cache_workspace_bytes(own, 1, 8) > 0 and binding.g10_cache_shared_workspace_bytes(own, 1, 8) > 0
    assert binding.g10_packed_workspace_bytes(theirs, 1, 8) > 0
    for call, cache in ((binding.g10_cache_workspace_bytes, theirs), (binding.g10_cache_shared_workspace_bytes, theirs), (binding.g10_packed_workspace_bytes, own)):
        with pytest.raises(binding.G10Error, match="takes a"):
            call(cache, 1, 8)
