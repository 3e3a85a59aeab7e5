"""Calls on the cache of 8-bit rows that are refused before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

from paper_2310_09443_b200 import binding, build

FAKE = 1 << 20                                          # an address that is aligned; never followed


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def packed(code=0, scales=FAKE, **change):
    c = binding._Cache(0, 2, 4, 64, 16, 8, 100, FAKE, FAKE, 16 * 4 * 64, 4 * 64, 64, FAKE, 8, FAKE, None, FAKE, None, FAKE)
    for k, v in change.items():
        setattr(c, k, v)
    return C.byref(binding._Packed(c, code, scales))


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


def rows(**change):
    r = binding._PackedRows(4, FAKE, FAKE, FAKE, *(512, 256, 64) * 2)
    for k, v in change.items():
        setattr(r, k, v)
    return C.byref(r)


def plan(**change):
    p = binding._CachePlan(64, 4, 8, FAKE, FAKE, FAKE)
    for k, v in change.items():
        setattr(p, k, v)
    return C.byref(p)


BAD = [(dict(code=2), -1), (dict(code=-1), -1), (dict(dtype=2), -1), (dict(num_seqs=-1), -1), (dict(num_seqs=65536), -2), (dict(kv_heads=0), -1), (dict(kv_heads=1025), -2),
       (dict(head_dim=8), -1), (dict(head_dim=24), -1), (dict(head_dim=272), -2), (dict(page_size=0), -1), (dict(page_size=65537), -2), (dict(max_pages=-1), -1),
       (dict(max_pages=1 << 30), -2), (dict(num_pages=-1), -1), (dict(num_pages=1 << 31), -2), (dict(lengths=None), -1), (dict(page_table=None), -1),
       (dict(table_stride=7), -1), (dict(status=None), -1)]
BAD_ROWS = [(dict(k=None), -1), (dict(v=None), -1), (dict(k=FAKE + 8), -1), (dict(scales=None), -1), (dict(scales=FAKE + 4), -1), (dict(page_stride=4104), -1),
            (dict(slot_stride=264), -1), (dict(head_stride=72), -1), (dict(head_stride=-64), -1), (dict(page_stride=1 << 34), -2)]


@pytest.mark.parametrize("change,code", BAD + BAD_ROWS)
def test_caches(lib, change, code):
    out = C.c_size_t(0)
    assert lib.g10_packed_append(packed(**change), tokens(), None) == code
    assert lib.g10_packed_read(packed(**change), rows(), None) == code
    assert lib.g10_packed_attend(packed(**change), queries(), FAKE, 1 << 40, None) == code
    assert lib.g10_packed_evict(packed(**change), plan(), None) == code
    if (change, code) in BAD:
        assert lib.g10_packed_workspace_bytes(packed(**change), 1, 8, 0, 0, 0, C.byref(out)) == code


def test_null_arguments(lib):
    out = C.c_size_t(0)
    assert lib.g10_packed_append(None, tokens(), None) == -1 and lib.g10_packed_append(packed(), None, None) == -1
    assert lib.g10_packed_read(None, rows(), None) == -1 and lib.g10_packed_read(packed(), None, None) == -1
    assert lib.g10_packed_attend(None, queries(), FAKE, 1 << 40, None) == -1 and lib.g10_packed_attend(packed(), None, FAKE, 1 << 40, None) == -1
    assert lib.g10_packed_evict(None, plan(), None) == -1 and lib.g10_packed_evict(packed(), None, None) == -1
    assert lib.g10_packed_workspace_bytes(None, 1, 8, 0, 0, 0, C.byref(out)) == -1 and lib.g10_packed_workspace_bytes(packed(), 1, 8, 0, 0, 0, None) == -1


@pytest.mark.parametrize("change,code", [(dict(tokens=-1), -1), (dict(k=FAKE + 8), -1), (dict(v=FAKE + 2), -1), (dict(k_seq_stride=4), -1), (dict(k_token_stride=63), -1),
                                         (dict(v_head_stride=65), -1), (dict(tokens=(1 << 31) - 1), -2)])
def test_rows(lib, change, code):
    assert lib.g10_packed_read(packed(), rows(**change), None) == code


@pytest.mark.parametrize("change,code", [(dict(new_tokens=0), -1), (dict(q_heads=0), -1), (dict(q_heads=6), -1), (dict(window=-1), -1), (dict(sinks=-1), -1),
                                         (dict(new_tokens=513), -2), (dict(q=None), -1), (dict(out=FAKE + 8), -1), (dict(q_head_stride=4), -1),
                                         (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1)])
def test_queries(lib, change, code):
    assert lib.g10_packed_attend(packed(), queries(**change), FAKE, 1 << 40, None) == code


def test_attend_wants_its_workspace_scores_and_no_positions_with_a_window(lib):
    out = C.c_size_t(0)
    assert lib.g10_packed_workspace_bytes(packed(), 1, 8, 0, 0, 1, C.byref(out)) == 0
    for ws, n in ((None, 1 << 40), (FAKE + 8, 1 << 40), (FAKE, out.value - 1)):
        assert lib.g10_packed_attend(packed(), queries(add_scores=1), ws, n, None) == -3
    assert lib.g10_packed_attend(packed(scores=None), queries(add_scores=1), FAKE, 1 << 40, None) == -1
    assert lib.g10_packed_attend(packed(positions=FAKE), queries(window=5), FAKE, 1 << 40, None) == -1


@pytest.mark.parametrize("change", [dict(new_tokens=0), dict(q_heads=-1), dict(rotary_dim=3), dict(rotary_dim=66), dict(rotary_dim=32), dict(k=None), dict(v=FAKE + 8),
                                    dict(k_token_stride=4), dict(q=None), dict(q_out=FAKE + 8), dict(q_weight=FAKE + 2)])
def test_tokens(lib, change):
    assert lib.g10_packed_append(packed(), tokens(**change), None) == -1


@pytest.mark.parametrize("change,code", [(dict(budget=0), -1), (dict(budget=(1 << 31) - 1), -2), (dict(moves=None), -1), (dict(counts=None), -1), (dict(moves=FAKE + 4), -1)])
def test_plans(lib, change, code):
    assert lib.g10_packed_evict(packed(), plan(**change), None) == code


def test_nothing_to_do(lib):
    assert lib.g10_packed_append(packed(num_seqs=0), tokens(), None) == 0
    assert lib.g10_packed_attend(packed(num_seqs=0), queries(), None, 0, None) == 0
    assert lib.g10_packed_evict(packed(num_seqs=0), plan(), None) == 0
    assert lib.g10_packed_read(packed(num_seqs=0), rows(), None) == 0
    assert lib.g10_packed_read(packed(), rows(tokens=0), None) == 0
    assert lib.g10_packed_read(packed(), rows(k=None, v=None), None) == 0


def test_attend_behind_a_shared_beginning(lib):
    out = C.c_size_t(0)
    cache = lambda **change: C.byref(packed(**change)._obj.cache)
    bytes_of = lambda c, *more: lib.g10_cache_shared_workspace_bytes(c, *more, C.byref(out))
    call = lambda c, u=None, shared=FAKE, ws=FAKE, n=1 << 40: lib.g10_cache_attend_shared(c, u or queries(), shared, ws, n, None)
    assert bytes_of(cache(), 1, 8) == 0
    for ws, n in ((None, 1 << 40), (FAKE + 8, 1 << 40), (FAKE, out.value - 1)):
        assert call(cache(), ws=ws, n=n) == -3
    assert call(cache(), shared=None) == -1 and call(None) == -1 and call(cache(dtype=3)) == -1
    for change, code in ((dict(window=4), -1), (dict(add_scores=1), -1), (dict(q=None), -1), (dict(new_tokens=0), -1), (dict(q_heads=6), -1), (dict(new_tokens=513), -2),
                         (dict(scale=float("nan")), -1)):
        assert call(cache(), queries(**change)) == code
    assert call(cache(num_seqs=0)) == 0
    assert bytes_of(cache(), 0, 8) == -1 and bytes_of(cache(), 1, 6) == -1 and bytes_of(cache(num_seqs=65535), 512, 8) == 0
    assert lib.g10_cache_shared_workspace_bytes(cache(), 1, 8, None) == -1
