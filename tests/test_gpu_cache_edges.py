"""The key-value cache on the device at the edges of what its calls allow, against the definitions in 64 bits (cache_oracle.py)."""
import math
import time
from types import SimpleNamespace

import pytest
import torch

import cache_oracle as O
from test_gpu_cache import DEV, check_attend, check_plan_and_evict, g10, queries, same, shuffle_positions  # noqa: F401 (g10 is the fixture)

pytestmark = pytest.mark.gpu


# ---- weights far below the largest -------------------------------------------------------------------------------------
@pytest.mark.parametrize("below", [10.0, 16.0, 17.5, 21.0])
@pytest.mark.parametrize("where", [0, 6_000, 12_002])
@pytest.mark.parametrize("group", [4, 20])
def test_many_weights_far_below_one(g10, below, where, group):
    """One slot with a value of zero outweighs each of 12 002 equal ones with a value of one by e^below: the answer is what these add up to.  So many
    heads that a block goes through whole sequences, and has that slot and thousands of the others under one maximum.

    The bound is that of attend_bounds with 2^-35 of the row's largest weight in place of half the smallest fp16 subnormal: fp16 weights are kept
    2^10 times too large (a weight of 1 then is 2^10, so half a subnormal step, 2^-25, is 2^-35 of the largest)."""
    n, kv = 12_003, 640
    c = O.make_cache([n], kv, 8, 64, torch.float16, 1, scores=False)
    pg, pl = O.places(c, 0, n)
    c.k[pg, pl], c.v[pg, pl] = 0.0, 1.0
    c.k[pg[where], pl[where], :, 0] = below
    c.v[pg[where], pl[where]] = 0.0
    q = torch.zeros(1, 1, kv * group, 8, dtype=torch.float16)
    q[..., 0] = 1.0
    lse = torch.empty(q.shape[:3], device=DEV)
    cache = O.upload(g10, c)
    out = g10.g10_cache_attend(cache, q.to(DEV), scale=1.0, lse=lse).cpu().double()
    assert int(cache.status.item()) == 0
    one = SimpleNamespace(**{**vars(c), "k": c.k[:, :, :1], "v": c.v[:, :, :1], "kv_heads": 1})        # (all heads are alike)
    r = O.attend(one, q[:, :, :1], 1.0)
    b_out, b_lse, _ = O.attend_bounds(one, r)
    b_out = b_out - (2.0 ** -25 - 2.0 ** -35) * r.all_v
    off = (out - r.out).abs() - b_out
    assert (off <= 0).all(), "%g instead of %g, off by %g over the bound" % (out.flatten()[off.argmax()], r.out.flatten()[0], off.max())
    assert ((lse.cpu().double() - r.lse).abs() <= b_lse).all()


@pytest.mark.parametrize("new,group", [(1, 4), (1, 12), (30, 4)])
def test_large_fp16_values_under_lifted_weights(g10, new, group):
    """Values at the type's end, the largest weights as large as they get: nothing overflows on the way to sums that are in range."""
    c = O.make_cache([2000, new + 3], 2, 64, 16, torch.float16, 4)
    own = torch.isfinite(c.v)
    c.v[own] = torch.where(c.v[own] > 0, 65504.0, 65000.0).half()
    q = queries(c, new, group, 2)
    # (k along q's first element rises a little less than the reference's slack from tile to tile)
    for s, n in enumerate(c.lengths.tolist()):
        pg, pl = O.places(c, s, n)
        c.k[pg, pl] = 0.0
        c.k[pg, pl, :, 0] = (torch.arange(n)[:, None] * 0.02).half()
    q[:] = 0.0
    q[..., 0] = 1.0
    check_attend(g10, c, q, scale=1.0, book=True)


# ---- append ------------------------------------------------------------------------------------------------------------
def test_append_of_more_than_2_to_the_30_tokens(g10):
    """Offsets in 64 bits from the token's number on: 2^30 + 9 tokens of one head of 8 dims (16 GiB of keys), the values one row by a stride of zero."""
    n, page = (1 << 30) + 9, 65536
    pages = -(-n // page)
    torch.cuda.empty_cache()
    k = torch.zeros(1, n, 1, 8, dtype=torch.bfloat16, device=DEV)
    there = [0, 1, 7, 8, 12345, n // 2, n - 18, n - 17, n - 10, n - 9, n - 8, n - 2, n - 1]
    for t in there:
        k[0, t] = torch.randn(8, dtype=torch.bfloat16, device=DEV)
    v = torch.randn(1, 1, 1, 8, dtype=torch.bfloat16, device=DEV).expand(1, n, 1, 8)
    pool_k, pool_v = (torch.zeros(pages, page, 1, 8, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cache = g10.CacheBuffers(pool_k, pool_v, torch.arange(pages, dtype=torch.int32, device=DEV)[None], torch.tensor([n], dtype=torch.int32, device=DEV))
    g10.g10_cache_append(cache, k, v)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    rows_k, rows_v = pool_k.view(-1, 8), pool_v.view(-1, 8)
    assert all(same(rows_k[t], k[0, t, 0]) and same(rows_v[t], v[0, 0, 0]) for t in there)
    step = 1 << 26
    for t in range(0, n, step):
        m = min(step, n - t)
        assert torch.equal(rows_k[t:t + m], k[0, t:t + m, 0]) and bool((rows_v[t:t + m] == v[0, 0, 0]).all())
    assert not rows_k[n:].any() and not rows_v[n:].any()
    # padding that far behind the tokens that count
    pool_k.zero_()
    g10.g10_cache_append(cache, k, v, counts=torch.tensor([3], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    assert same(rows_k[n - 3:n], k[0, :3, 0]) and not rows_k[:1 << 20].any()
    del k, v, pool_k, pool_v, rows_k, rows_v, cache
    torch.cuda.empty_cache()


# ---- tables without columns, pools without pages ----------------------------------------------------------------------
@pytest.mark.parametrize("new,group", [(1, 2), (1, 12), (4, 6)])
@pytest.mark.parametrize("pages", [0, 3])
@pytest.mark.parametrize("columns", [0, 2])
def test_nothing_to_look_at(g10, new, group, pages, columns):
    """Before the first page is given out.  Lengths of zero; or, where there are columns, lengths whose pages are none: read as zeros."""
    on = dict(device=DEV)
    k = torch.randn(pages, 16, 2, 64, **on).to(torch.bfloat16)
    cells = (pages, 2, 16)
    scores, positions = torch.rand(cells, **on), torch.zeros(cells, dtype=torch.int32, **on)
    before = [x.clone() for x in (k, scores)]
    table = torch.full((3, columns), -1, dtype=torch.int32, **on)
    for lengths in ([0, 0, 0],) if columns == 0 else ([0, 0, 0], [0, 5, 32]):
        cache = g10.CacheBuffers(k, k.clone(), table, torch.tensor(lengths, dtype=torch.int32, **on), scores=scores, positions=positions)
        q = torch.randn(3, new, 2 * group, 64, **on).to(torch.bfloat16)
        out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:3], 9.0, **on)
        g10.g10_cache_attend(cache, q, add_scores=True, out=out, lse=lse)
        rows = torch.randn(3, new, 2, 64, **on).to(torch.bfloat16)
        q_out = g10.g10_cache_append(cache, rows, rows, q)
        p = g10.g10_cache_plan_evictions(cache, 4, 1, 1)
        g10.g10_cache_evict(cache, p.moves, p.counts)
        torch.cuda.synchronize()
        assert int(cache.status.item()) == (0x400 if any(lengths) else 0)
        assert not out.any() and p.new_lengths.tolist() == [min(n, 4) for n in lengths]
        for s, n in enumerate(lengths):
            count = min(n, new)
            assert not q_out[s, count:].any() and same(q_out[s, :count], q[s, :count])
            for t in range(new):
                want = math.log(n - count + t + 1) if t < count else -math.inf
                assert torch.allclose(lse[s, t].double().cpu(), torch.tensor(want, dtype=torch.float64), rtol=2.0 ** -20, atol=2.0 ** -20)
        assert same(k, before[0]) and same(scores, before[1])


# ---- the status word -----------------------------------------------------------------------------------------------------
def test_a_status_word_made_here_is_cleared_before_the_first_call(g10):
    """Work that waits on the current stream does not clear it after a call on another stream has written to it."""
    c = O.make_cache([40, 40], 2, 64, 16, torch.bfloat16, 3, scores=False)
    k, v, table = c.k.to(DEV), c.v.to(DEV), c.table.to(DEV)
    lengths = torch.tensor([40, 49], dtype=torch.int32, device=DEV)          # (49: more than the table has room for)
    q = queries(c, 1, 2, 1).to(DEV)
    side = torch.cuda.Stream()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device=DEV)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    word = torch.zeros(1, dtype=torch.int64, device=DEV)
    g10.g10_cache_attend(g10.CacheBuffers(k, v, table, lengths, status=word), q, out=out, lse=lse, ws=ws, stream=side)      # (all is loaded)
    torch.cuda.synchronize()
    torch.cuda._sleep(40_000_000)
    cache = g10.CacheBuffers(k, v, table, lengths)
    g10.g10_cache_attend(cache, q, out=out, lse=lse, ws=ws, stream=side)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0x800


def test_the_tensors_of_a_cache_are_fixed(g10):
    """An assignment would leave the calls with the old tensor's address: it is refused; writing into the tensor is what counts."""
    c = O.make_cache([40, 30], 1, 64, 16, torch.bfloat16, 3, positions=True)
    cache = O.upload(g10, c)
    for name in ("k", "v", "page_table", "lengths", "seen", "scores", "positions", "status"):
        old = getattr(cache, name)
        with pytest.raises(g10.G10Error, match=name):
            setattr(cache, name, torch.zeros(2, dtype=torch.int32, device=DEV))
        assert getattr(cache, name) is old
    lengths = cache.lengths
    lengths -= 10
    cache.lengths -= 1
    assert g10.g10_cache_plan_evictions(cache, 25).new_lengths.tolist() == [25, 19]
    cache.layer = 7                                      # (whatever else a program keeps there)


# ---- numbers of more than 32 bits ------------------------------------------------------------------------------------------
def test_numbers_that_do_not_fit_are_refused(g10):
    """A window of 2^32 + 5 is not one of 5."""
    c = O.make_cache([40], 1, 64, 16, torch.bfloat16, 3)
    cache = O.upload(g10, c)
    big = 2 ** 32 + 5
    q = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    kv = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16, device=DEV)
    many = kv.expand(1, big, 1, 64)
    before = [x.clone() for x in (cache.k, cache.v, cache.scores)]
    calls = [lambda: g10.g10_cache_attend(cache, q, window=big), lambda: g10.g10_cache_attend(cache, q, window=4, sinks=big),
             lambda: g10.g10_cache_attend(cache, q, window=-2 ** 32 + 5), lambda: g10.g10_cache_workspace_bytes(cache, 1, 2, window=big),
             lambda: g10.g10_cache_workspace_bytes(cache, big, 2), lambda: g10.g10_cache_append(cache, many, many),
             lambda: g10.g10_cache_plan_evictions(cache, 8, recent=2 ** 32), lambda: g10.g10_cache_plan_evictions(cache, 8, sinks=2 ** 32),
             lambda: g10.g10_cache_plan_evictions(cache, big)]
    for i, call in enumerate(calls):
        with pytest.raises(g10.G10Error, match="32 bits"):
            call()
            raise AssertionError("call %d was taken" % i)
    assert all(same(a, b) for a, b in zip(before, (cache.k, cache.v, cache.scores)))


# ---- forms that only large sizes take --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("lengths,columns,budget", [([3000, 70, 500, 0], 8000, 200), ([3000, 70, 500, 0], 8000, 2999), ([410_001, 9], None, 4000)])
def test_plan_where_shared_memory_holds_no_scores(g10, lengths, columns, budget):
    """Some 48 000 slots a block is what it takes: tables of half a million slots, long sequences and short ones."""
    c = O.make_cache(lengths, 2, 8, 64, torch.bfloat16, 7, columns=columns, positions=True)
    shuffle_positions(c, 3)
    check_plan_and_evict(g10, c, budget, 4, budget // 8)


@pytest.mark.parametrize("seqs,kv,dim,group,new", [(32, 16, 192, 2, 1), (32, 16, 256, 6, 2), (64, 16, 80, 1, 1), (128, 4, 64, 20, 1), (128, 4, 256, 9, 2)])
def test_shares_that_are_cut(g10, seqs, kv, dim, group, new):
    """At least 128 tiles for each block that runs at a time: four shares for each.  The sequences have the same pages, so that it takes little memory;
    what is booked adds up."""
    lengths = [2560 - i for i in range(seqs)]
    c = O.make_cache(lengths[:1], kv, dim, 64, torch.bfloat16, dim)
    c.lengths = torch.tensor(lengths, dtype=torch.int32)
    c.table = c.table.expand(seqs, -1).contiguous()
    c.scores.zero_()
    q = queries(c, new, group, 4)
    cache = O.upload(g10, c)
    lse = torch.empty(q.shape[:3], device=DEV)
    out = g10.g10_cache_attend(cache, q.to(DEV), add_scores=True, lse=lse).cpu().double()
    assert int(cache.status.item()) == 0
    r = O.attend(c, q, dim ** -0.5)
    b_out, b_lse, rel = O.attend_bounds(c, r)
    assert ((out - r.out).abs() <= b_out).all() and ((lse.cpu().double() - r.lse).abs() <= b_lse).all()
    got, want = cache.scores.cpu().double(), torch.zeros(c.scores.shape, dtype=torch.float64)
    for (s, h), w in r.booked.items():
        pg, pl = O.places(c, s, len(w))
        want[pg, h, pl] += w
    # (one rounded addition for each sequence)
    assert ((got - want).abs() <= want * (float(rel.max()) * 1.01 + seqs * 2.0 ** -24)).all()


def test_evict_of_more_heads_than_one_launch_takes(g10):
    """1100 sequences of 64 heads: 70 400 pairs, 65 472 in the first launch."""
    lengths = [6 + i % 3 if i % 2 == 0 or i > 1000 else i % 5 for i in range(1100)]
    c = O.make_cache(lengths, 64, 8, 4, torch.float16, 2, positions=True)
    check_plan_and_evict(g10, c, 5, 1, 1)


def test_a_prompt_in_parts(g10):
    """More tokens than one call takes: parts with lengths of their own give what the definitions give for the whole, booked weights too."""
    prompts, group, part = [700, 333], 4, 256
    c = O.make_cache([n + 50 for n in prompts], 2, 64, 16, torch.bfloat16, 9)
    q = queries(c, 700, group, 5)
    counts = torch.tensor(prompts, dtype=torch.int32)
    r = O.attend(c, q, 0.125, counts=counts)
    cache = O.upload(g10, c)
    dq, lengths = q.to(DEV), cache.lengths
    with pytest.raises(g10.G10Error):
        g10.g10_cache_attend(cache, dq, counts=counts.to(DEV))
    ends = lengths.clone()
    view = g10.CacheBuffers(cache.k, cache.v, cache.page_table, ends, scores=cache.scores, status=cache.status)
    done = counts.to(DEV)
    outs = []
    for t in range(0, 700, part):
        mine = (done - t).clamp(0, part).int()
        ends.copy_(lengths - done + (done.clamp(max=t + part)))
        outs.append(g10.g10_cache_attend(view, dq[:, t:t + part], scale=0.125, counts=mine, add_scores=True))
    out = torch.cat(outs, 1).cpu().double()
    assert int(cache.status.item()) == 0
    bound, _, rel = O.attend_bounds(c, r)
    assert ((out - r.out).abs() <= bound).all()
    got = cache.scores.cpu().double()
    for (s, h), w in r.booked.items():
        pg, pl = O.places(c, s, len(w))
        was = c.scores[pg, h, pl].double()
        # (three additions to a score, each rounded)
        assert ((got[pg, h, pl] - was - w).abs() <= w * float(rel[s].max()) * 1.01 + 3 * 2.0 ** -24 * (was + w)).all()


# ---- what is wrong in the data, for many rows ------------------------------------------------------------------------------------
@pytest.mark.parametrize("new,group", [(1, 20), (20, 7)])
@pytest.mark.parametrize("book", [False, True])
def test_bad_pages_and_lengths_for_many_rows(g10, new, group, book):
    """Reported; a slot without a page is read as zeros and not written, a length is taken as the nearest that is possible."""
    c = O.make_cache([200, 190], 2, 64, 16, torch.bfloat16, 3)
    c.table = torch.cat([c.table, c.table[:, :1]], 1).contiguous()           # (room for more slots than there are)
    c.table[:, -1] = c.table[0, 0]
    q = queries(c, new, group, 1)
    dq = q.to(DEV)
    good = c.table.clone()
    capacity = 16 * c.table.shape[1]

    def call(counts=None):
        cache = O.upload(g10, c)
        out = g10.g10_cache_attend(cache, dq, scale=0.1, add_scores=book, counts=counts)
        torch.cuda.synchronize()
        assert same(cache.k, c.k) and same(cache.v, c.v)
        return cache, out.cpu().double()

    for page in (-1, -2 ** 31, c.k.shape[0], 2 ** 31 - 1):
        c.table[1, 2] = page
        cache, out = call()
        assert int(cache.status.item()) == 0x400
        # the same with a page of zeros there: the one that nobody has
        spare = next(i for i in range(c.k.shape[0]) if i not in good.flatten().tolist())
        c.table[1, 2] = spare
        kept = c.k[spare].clone(), c.v[spare].clone(), c.scores[spare].clone()
        c.k[spare], c.v[spare] = 0.0, 0.0
        r = O.attend(c, q, 0.1)
        bound = O.attend_bounds(c, r)[0]
        assert ((out - r.out).abs() <= bound).all()
        if book:
            got = cache.scores.cpu()
            assert same(got[spare], kept[2])
            pg, pl = O.places(c, 1, 190)
            for h in range(2):
                want = c.scores[pg, h, pl].double() + r.booked[1, h]
                there = pg != spare
                assert ((got[pg, h, pl].double() - want).abs() <= want * 0.001)[there].all()
        c.k[spare], c.v[spare] = kept[0], kept[1]
        c.table[1, 2] = good[1, 2]
    for length, nearest in ((-1, 0), (-2 ** 31, 0), (capacity + 1, capacity), (2 ** 31 - 1, capacity)):
        c.lengths[1] = length
        cache, out = call()
        c.lengths[1] = nearest
        again, want = call()
        # (all that the table has room for: one entry of this sequence's names no page)
        assert int(again.status.item()) == (0x400 if nearest else 0) and int(cache.status.item()) == int(again.status.item()) | 0x800
        assert same(out.float(), want.float())
    c.lengths[1] = 190
    for count, nearest in ((-1, 0), (new + 1, new), (2 ** 31 - 1, new)):
        cache, out = call(torch.tensor([new, count], dtype=torch.int32, device=DEV))
        assert int(cache.status.item()) == 0x800
        again, want = call(torch.tensor([new, nearest], dtype=torch.int32, device=DEV))
        assert int(again.status.item()) == 0 and same(out.float(), want.float())


# ---- waits that run out ------------------------------------------------------------------------------------------------
@pytest.fixture
def hooks(monkeypatch):
    """The test build of the library (-DG10_TEST_HOOKS), in which an environment variable names an arrival that the first block of the kernels for many rows
    keeps to itself; that block's waits are short."""
    from paper_2310_09443_b200 import binding, build
    monkeypatch.setattr(binding, "LIB_PATH", build.build(hooks=True))
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.delenv("G10_TEST_CACHE_MUTE", raising=False)
    binding.load_library()
    return binding


@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("new,group", [(1, 20), (20, 8)])
def test_a_wait_that_runs_out(hooks, monkeypatch, dim, new, group):
    """A tile that is never told full, weights, logits, queries or room for logits that are never told of, in either kernel: the block gives up, the call
    returns with the timeout bit, nothing is written out of place, and the next call is right.  Nothing traps, faults or spins on."""
    c = O.make_cache([9000, 700, 2500 + new], 8, dim, 64, torch.bfloat16, dim + group)
    q = queries(c, new, group, 3)
    dq = q.to(DEV)
    r = O.attend(c, q, dim ** -0.5)
    bound, _, rel = O.attend_bounds(c, r)
    around = torch.full((2 * dq.numel(),), 7.0, dtype=dq.dtype, device=DEV)
    out = around[dq.numel() // 2:][:dq.numel()].view(dq.shape)
    size = hooks.g10_cache_workspace_bytes(O.upload(hooks, c), new, 8 * group, add_scores=True)
    ws = torch.zeros(size + 1024, dtype=torch.uint8, device=DEV)
    for mute in (0, 1, 2, 3, 4, 5, 6, 0):
        monkeypatch.setenv("G10_TEST_CACHE_MUTE", str(mute))
        cache = O.upload(hooks, c)
        t0 = time.perf_counter()
        hooks.g10_cache_attend(cache, dq, out=out, ws=ws[:size], add_scores=True)
        torch.cuda.synchronize()
        took = time.perf_counter() - t0
        assert int(cache.status.item()) == (0 if mute == 0 else 0x80), mute
        assert took < 1.0, (mute, took)
        assert (around[:dq.numel() // 2] == 7).all() and (around[dq.numel() // 2 + dq.numel():] == 7).all() and not ws[size:].any()
        assert same(cache.k, c.k) and same(cache.v, c.v)
        if mute == 0:
            assert ((out.cpu().double() - r.out).abs() <= bound).all()
            got = cache.scores.cpu()
            for (s, h), w in r.booked.items():
                pg, pl = O.places(c, s, len(w))
                was = c.scores[pg, h, pl].double()
                assert ((got[pg, h, pl].double() - was - w).abs() <= w * float(rel[s].max()) * 1.01 + 2.0 ** -23 * (was + w)).all()
