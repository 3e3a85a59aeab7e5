"""Calls on the key-value cache that are refused before anything is launched (no GPU needed): the C entry points with sizes and pointers
that no device would be given."""
import ctypes as C

import pytest

from paper_2310_09443_b200 import binding, build

FAKE = 1 << 20                                          # an address that is aligned; never followed


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def cache(**change):
    c = binding._Cache(0, 2, 4, 64, 16, 8, 100, FAKE, FAKE, 16 * 4 * 64, 4 * 64, 64, FAKE, 8, FAKE, None, FAKE, None, FAKE)
    for k, v in change.items():
        setattr(c, k, v)
    return C.byref(c)


BAD_CACHES = [(dict(dtype=2), -1), (dict(dtype=-1), -1), (dict(num_seqs=-1), -1), (dict(num_seqs=65536), -2), (dict(kv_heads=0), -1), (dict(kv_heads=1025), -2),
              (dict(head_dim=0), -1), (dict(head_dim=20), -1), (dict(head_dim=264), -2), (dict(page_size=0), -1), (dict(page_size=65537), -2),
              (dict(max_pages=-1), -1), (dict(max_pages=1 << 30), -2), (dict(num_pages=-1), -1), (dict(num_pages=1 << 31), -2), (dict(lengths=None), -1),
              (dict(page_table=None), -1), (dict(table_stride=7), -1), (dict(status=None), -1)]
BAD_ROWS = [dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(page_stride=4), dict(slot_stride=260), dict(head_stride=65)]


def queries(**change):
    u = binding._CacheQueries(1, 8, FAKE, 512, 512, 64, None, FAKE, None, 0.125, 0, 0, 0)
    for k, v in change.items():
        setattr(u, k, v)
    return C.byref(u)


def tokens(**change):
    t = binding._CacheTokens(1, 8, FAKE, FAKE, FAKE, *(512, 512, 64) * 3, FAKE, None, None, None, 1e-6, None, None, 0, 0, 0)
    for k, v in change.items():
        setattr(t, k, v)
    return C.byref(t)


def plan(**change):
    p = binding._CachePlan(64, 4, 8, FAKE, FAKE, FAKE)
    for k, v in change.items():
        setattr(p, k, v)
    return C.byref(p)


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_caches(lib, change, code):
    out = C.c_size_t(0)
    assert lib.g10_cache_append(cache(**change), tokens(), None) == code
    assert lib.g10_cache_attend(cache(**change), queries(), FAKE, 1 << 40, None) == code
    assert lib.g10_cache_plan_evictions(cache(**change), plan(), None) == code
    assert lib.g10_cache_evict(cache(**change), plan(), None) == code
    assert lib.g10_cache_workspace_bytes(cache(**change), 1, 8, 0, 0, 0, C.byref(out)) == code


@pytest.mark.parametrize("change", BAD_ROWS)
def test_rows(lib, change):
    assert lib.g10_cache_append(cache(**change), tokens(), None) == -1
    assert lib.g10_cache_attend(cache(**change), queries(), FAKE, 1 << 40, None) == -1
    assert lib.g10_cache_evict(cache(**change), plan(), None) == -1


@pytest.mark.parametrize("change,code", [(dict(new_tokens=0), -1), (dict(q_heads=0), -1), (dict(q_heads=6), -1), (dict(new_tokens=513), -2), (dict(q=None), -1),
                                         (dict(out=None), -1), (dict(q=FAKE + 4), -1), (dict(out=FAKE + 4), -1), (dict(q_seq_stride=4), -1),
                                         (dict(q_token_stride=4), -1), (dict(q_head_stride=4), -1), (dict(window=-1), -1), (dict(sinks=-1), -1),
                                         (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1), (dict(scale=3e38), -1), (dict(scale=-3e38), -1)])
def test_queries(lib, change, code):
    assert lib.g10_cache_attend(cache(), queries(**change), FAKE, 1 << 40, None) == code


def test_attend_wants_what_it_uses(lib):
    out = C.c_size_t(0)
    assert lib.g10_cache_attend(cache(), None, FAKE, 1 << 40, None) == -1
    assert lib.g10_cache_attend(cache(scores=None), queries(add_scores=1), FAKE, 1 << 40, None) == -1
    assert lib.g10_cache_attend(cache(positions=FAKE), queries(window=5), FAKE, 1 << 40, None) == -1
    assert lib.g10_cache_workspace_bytes(cache(), 1, 8, 0, 0, 1, C.byref(out)) == 0
    booked = out.value
    assert lib.g10_cache_workspace_bytes(cache(), 1, 8, 0, 0, 0, C.byref(out)) == 0
    assert 0 < out.value < booked and out.value % 256 == 0
    assert lib.g10_cache_workspace_bytes(cache(), 1, 8, 0, 0, 0, None) == -1
    assert lib.g10_cache_attend(cache(), queries(), None, out.value, None) == -3
    assert lib.g10_cache_attend(cache(), queries(), FAKE + 16, out.value, None) == -3
    assert lib.g10_cache_attend(cache(), queries(), FAKE, out.value - 1, None) == -3
    # a window needs no more than the whole cache does, and less of a long one
    assert lib.g10_cache_workspace_bytes(cache(max_pages=100000, table_stride=100000), 1, 8, 0, 0, 1, C.byref(out)) == 0
    whole = out.value
    assert lib.g10_cache_workspace_bytes(cache(max_pages=100000, table_stride=100000), 1, 8, 512, 4, 1, C.byref(out)) == 0
    assert out.value < whole / 2


@pytest.mark.parametrize("change", [dict(new_tokens=0), dict(q_heads=-1), dict(rotary_dim=-2), dict(rotary_dim=3), dict(rotary_dim=66), dict(rotary_dim=32),
                                    dict(rotary_dim=32, cos_table=FAKE), dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(k=FAKE + 8),
                                    dict(q_out=FAKE + 8), dict(k_token_stride=12), dict(v_seq_stride=12), dict(q_head_stride=12), dict(q_weight=FAKE + 2),
                                    dict(k_weight=FAKE + 2), dict(q_weight=FAKE, eps=-1.0), dict(k_weight=FAKE, eps=float("nan"))])
def test_tokens(lib, change):
    assert lib.g10_cache_append(cache(), tokens(**change), None) == -1


def test_token_limits(lib):
    assert lib.g10_cache_append(cache(), None, None) == -1
    assert lib.g10_cache_append(cache(num_seqs=65535), tokens(new_tokens=1 << 20), None) == -2


@pytest.mark.parametrize("change,code", [(dict(budget=0), -1), (dict(budget=-5), -1), (dict(sinks=-1), -1), (dict(recent=-1), -1), (dict(sinks=60, recent=5), -1),
                                         (dict(moves=None), -1), (dict(counts=None), -1), (dict(moves=FAKE + 4), -1), (dict(budget=0x7fffffff), -2)])
def test_plans(lib, change, code):
    assert lib.g10_cache_plan_evictions(cache(), plan(**change), None) == code
    if not {"sinks", "recent"} & set(change):
        assert lib.g10_cache_evict(cache(), plan(**change), None) == code


def test_plan_wants_scores(lib):
    assert lib.g10_cache_plan_evictions(cache(scores=None), plan(), None) == -1
    assert lib.g10_cache_plan_evictions(cache(), None, None) == -1 and lib.g10_cache_evict(cache(), None, None) == -1


def test_nothing_to_do_without_sequences(lib):
    """No launch at all, and no pointer is asked for."""
    empty = dict(num_seqs=0, lengths=None, page_table=None)
    assert lib.g10_cache_append(cache(**empty), tokens(), None) == 0
    assert lib.g10_cache_attend(cache(**empty), queries(q=None, out=None), None, 0, None) == 0
    assert lib.g10_cache_plan_evictions(cache(**empty), plan(moves=None), None) == 0
    assert lib.g10_cache_evict(cache(**empty), plan(moves=None), None) == 0


def test_binding_refuses_tensors_of_the_host():
    import torch
    z = torch.zeros(1, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(binding.G10Error):
        binding.CacheBuffers(z, z, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
