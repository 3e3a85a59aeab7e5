"""The key-value cache on the device against the definitions in 64 bits (cache_oracle.py)."""
import math

import numpy as np
import pytest
import torch

import cache_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def g10():
    from paper_2310_09443_b200 import binding, build
    build.build()
    binding.load_library()
    return binding


def same(a, b):
    """Equal bit for bit, NaN included."""
    kind = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.contiguous().view(kind).cpu(), b.contiguous().view(kind).cpu())


def check_attend(g10, c, q, window=0, sinks=0, counts=None, book=False, lse=True, scale=None, strided=False):
    scale = c.head_dim ** -0.5 if scale is None else scale
    cache = O.upload(g10, c)
    dq = q.to(DEV)
    if strided:
        wide = torch.full(q.shape[:2] + (q.shape[2] + 3, q.shape[3]), math.nan, dtype=q.dtype, device=DEV)
        wide[:, :, 1:-2] = dq
        dq = wide[:, :, 1:-2]
    got_lse = torch.full(q.shape[:3], 99.0, device=DEV) if lse else None
    out = torch.full(q.shape, 99.0, dtype=q.dtype, device=DEV)
    dc = None if counts is None else counts.to(DEV)
    g10.g10_cache_attend(cache, dq, scale=scale, window=window, sinks=sinks, counts=dc, add_scores=book, out=out, lse=got_lse)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    r = O.attend(c, q, scale, window, sinks, counts)
    b_out, b_lse, rel = O.attend_bounds(c, r)
    out = out.cpu().double()
    nothing = torch.isinf(r.lse)
    assert torch.isfinite(out).all()
    assert (out[nothing] == 0).all()
    off = (out - r.out).abs() - b_out
    assert off.max() <= 0, "out off by %g over the bound at %s" % (off.max(), np.unravel_index(int(off.argmax()), off.shape))
    if lse:
        got = got_lse.cpu().double()
        assert torch.equal(torch.isinf(got), nothing)
        assert ((got - r.lse).abs() <= b_lse)[~nothing].all()
    if book:
        new = cache.scores.cpu()
        want = c.scores.double().clone()
        slack = torch.zeros_like(want)
        for (s, h), w in r.booked.items():
            pg, pl = O.places(c, s, len(w))
            want[pg, h, pl] += w
            slack[pg, h, pl] = w * float(rel[s].max()) * 1.01 + 1e-30
        slack += 2.0 ** -23 * want.abs()
        assert ((new.double() - want).abs() <= slack).all()
        touched = want != c.scores.double()
        assert same(new[~touched], c.scores[~touched])
    elif c.scores is not None:
        assert same(cache.scores, c.scores)
    return cache


def queries(c, new, group, seed, spread=2.0):
    gen = torch.Generator().manual_seed(seed + 77)
    return (spread * torch.randn(len(c.lengths), new, c.kv_heads * group, c.head_dim, generator=gen)).to(c.dtype)


@pytest.mark.parametrize("dim", [8, 24, 64, 72, 80, 96, 128, 136, 192, 256])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_attend_head_dims(g10, dim, kind):
    c = O.make_cache([0, 1, 63, 64, 65, 200], 2, dim, 16, O.TYPES[kind], dim)
    check_attend(g10, c, queries(c, 1, 4, dim), book=True)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 15, 16, 17, 20, 40])
@pytest.mark.parametrize("book", [False, True])
def test_attend_groups(g10, group, book):
    c = O.make_cache([7, 129, 300, 0, 31], 3, 64, 8, torch.bfloat16, group)
    check_attend(g10, c, queries(c, 1, group, group), book=book, strided=book)


@pytest.mark.parametrize("page", [1, 3, 7, 16, 48, 64, 100, 256])
@pytest.mark.parametrize("layout", ["slots", "heads", "wide"])
def test_attend_pages_and_strides(g10, page, layout):
    c = O.make_cache([1, 5, 97, 100, 101, 333], 2, 128, page, torch.float16, page, layout=layout)
    check_attend(g10, c, queries(c, 1, 4, page), book=True)


@pytest.mark.parametrize("new,group", [(2, 1), (3, 4), (5, 3), (16, 1), (16, 4), (9, 7), (33, 2), (70, 1), (16, 16), (130, 3)])
@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("fp16", 80)])
def test_attend_several_tokens(g10, new, group, kind, dim):
    lengths = [new + 61, new, 1, 0, new + 200, max(1, new // 2)]
    c = O.make_cache(lengths, 2, dim, 16, O.TYPES[kind], new * group)
    check_attend(g10, c, queries(c, new, group, new), book=True)
    counts = torch.tensor([new, max(1, new // 3), 1, 0, 0, new], dtype=torch.int32)
    check_attend(g10, c, queries(c, new, group, new + 1), book=True, counts=counts)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 5), (63, 0), (64, 64), (65, 1), (100, 70), (500, 3), (5000, 5000)])
@pytest.mark.parametrize("new,group", [(1, 4), (6, 1), (40, 2)])
def test_attend_window_and_sinks(g10, window, sinks, new, group):
    c = O.make_cache([1, 64, 130, 400, 777, 0], 2, 64, 24, torch.bfloat16, window)
    check_attend(g10, c, queries(c, new, group, sinks), window=window, sinks=sinks, book=True)


@pytest.mark.parametrize("dim", [8, 64, 80, 96, 128, 192, 256])
@pytest.mark.parametrize("group,new", [(1, 1), (4, 1), (7, 2), (16, 2), (3, 30)])
def test_attend_with_room_in_the_table(g10, dim, group, new):
    """Tables much longer than the sequences: what a block has to do is then not known before the lengths are read."""
    lengths = [new + 1, new + 700, 0, 1, new + 64, 330]
    for page, columns in ((16, 400), (64, 1000)):
        c = O.make_cache(lengths, 2, dim, page, torch.bfloat16, dim + group, columns=columns)
        check_attend(g10, c, queries(c, new, group, dim), book=True)
        check_attend(g10, c, queries(c, new, group, dim + 1), window=150, sinks=70)


@pytest.mark.parametrize("tiles", [1, 2, 3, 5, 8, 9, 16, 31, 32, 33])
@pytest.mark.parametrize("group", [1, 12])
def test_attend_lengths_about_what_a_cluster_takes(g10, tiles, group):
    for lengths in ([64 * tiles], [64 * tiles - 63, 0, 1], [64 * tiles, 64, 65, 64 * tiles - 1]):
        c = O.make_cache(lengths, 2, 128, 32, torch.float16, tiles)
        check_attend(g10, c, queries(c, 1, group, tiles), book=True)
        check_attend(g10, c, queries(c, 1, group, tiles), window=100, sinks=3)


def test_attend_window_reads_nothing_outside(g10):
    """What stands between the first slots and the window may be anything."""
    c = O.make_cache([700], 2, 64, 16, torch.float16, 3)
    pg, pl = O.places(c, 0, 700)
    for x in (c.k, c.v):
        x[pg[3:600], pl[3:600]] = math.nan
    check_attend(g10, c, queries(c, 1, 4, 1), window=100, sinks=3, book=True)
    check_attend(g10, c, queries(c, 5, 2, 1), window=96, sinks=3, book=True)


@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("new,group,window", [(4, 2, 0), (17, 3, 0), (5, 1, 30)])
def test_attend_later_tokens_may_be_anything(g10, what, new, group, window):
    """The rows before a token that is not finite are as if it was not there."""
    c = O.make_cache([150, new + 1], 2, 128, 16, torch.bfloat16, 9)
    q = queries(c, new, group, 5)
    clean = O.attend(c, q, 0.1, window)
    b_out, b_lse, _ = O.attend_bounds(c, clean)
    for s, n in enumerate(c.lengths.tolist()):
        pg, pl = O.places(c, s, n)
        c.k[pg[-1], pl[-1]] = what
        c.v[pg[-1], pl[-1], :, 1::3] = what
    cache = O.upload(g10, c)
    lse = torch.empty(q.shape[:3], device=DEV)
    out = g10.g10_cache_attend(cache, q.to(DEV), scale=0.1, window=window, lse=lse).cpu().double()
    assert ((out - clean.out).abs() <= b_out)[:, :-1].all()
    assert ((lse.cpu().double() - clean.lse).abs() <= b_lse)[:, :-1].all()


def test_attend_padding_rows_beside_values_that_are_not_finite(g10):
    c = O.make_cache([200, 90], 1, 64, 16, torch.float16, 4)
    pg, pl = O.places(c, 0, 200)
    c.v[pg[10], pl[10]] = math.inf
    q = queries(c, 3, 2, 6)
    counts = torch.tensor([1, 2], dtype=torch.int32)
    out = g10.g10_cache_attend(O.upload(g10, c), q.to(DEV), counts=counts.to(DEV)).cpu()
    assert (out[0, 1:] == 0).all() and (out[1, 2:] == 0).all()
    assert torch.isinf(out[0, 0]).all() and torch.isfinite(out[1, :2]).all()


def test_attend_spreads_and_extremes(g10):
    """Logits from nearly equal to one that outweighs all others, and a scale of zero."""
    c = O.make_cache([300, 999, 2], 2, 128, 16, torch.bfloat16, 21)
    for spread in (0.0, 0.01, 30.0):
        check_attend(g10, c, queries(c, 1, 8, 2, spread=spread), book=True)
    check_attend(g10, c, queries(c, 1, 8, 2), scale=0.0, book=True)
    check_attend(g10, c, queries(c, 1, 8, 2), scale=-0.2)


@pytest.mark.parametrize("new,group", [(1, 8), (1, 12), (5, 5), (30, 4), (2, 80)])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_attend_where_later_slots_outweigh_all_before(g10, new, group, kind):
    """Logits that rise along the sequence, by a little or by so much that each tile makes what was before it vanish; and that fall."""
    c = O.make_cache([1000, 130 + new], 2, 64, 16, O.TYPES[kind], 31)
    q = torch.ones(2, new, 2 * group, 64, dtype=c.dtype)
    q[:, :, 1::2] = -1
    for rise in (0.004, 0.05, 0.5):
        for s, n in enumerate(c.lengths.tolist()):
            pg, pl = O.places(c, s, n)
            c.k[pg, pl] = (torch.arange(n)[:, None, None] * rise / 64 + 0.01 * torch.randn(n, 2, 64, generator=torch.Generator().manual_seed(s))).to(c.dtype)
        for scale in (1.0, -1.0, 4.0, 0.0):
            check_attend(g10, c, q, scale=scale, book=True)


@pytest.mark.parametrize("lengths,kv,group,dim", [([9001], 1, 8, 128), ([20000, 3, 4000, 0, 900], 2, 4, 64), ([5000] * 40, 4, 1, 64), ([2500] * 7, 8, 16, 128), ([3000, 1], 1, 1, 256),
                                                  ([6000, 1, 2000], 2, 24, 128), ([3000] * 9, 3, 40, 96), ([4000, 70], 1, 200, 256)])
def test_attend_long(g10, lengths, kv, group, dim):
    c = O.make_cache(lengths, kv, dim, 64, torch.bfloat16, len(lengths))
    check_attend(g10, c, queries(c, 1, group, 3), book=True)


def test_attend_many_sequences(g10):
    """More sequences than threads of a block, most of them short or empty."""
    rng = np.random.default_rng(5)
    lengths = [int(x) for x in rng.integers(0, 40, size=1500)]
    c = O.make_cache(lengths, 1, 64, 8, torch.bfloat16, 8)
    check_attend(g10, c, queries(c, 1, 2, 8), book=True)


def test_attend_same_bits_each_time(g10):
    c = O.make_cache([4000, 100, 2222], 2, 128, 16, torch.bfloat16, 2)
    q = queries(c, 9, 4, 1).to(DEV)
    got = []
    for _ in range(3):
        cache = O.upload(g10, c)
        lse = torch.empty(q.shape[:3], device=DEV)
        got.append((g10.g10_cache_attend(cache, q, lse=lse, add_scores=True), lse, cache.scores))
    for x in got[1:]:
        for a, b in zip(x, got[0]):
            assert same(a, b)


def test_offsets_beyond_32_bits(g10):
    """Pages behind the first 2^32 elements of the pool, for every call."""
    page, kv, dim = 64, 2, 128
    pages = (1 << 32) // (page * kv * dim) + 8
    c = O.make_cache([130, 200], kv, dim, page, torch.bfloat16, 6, positions=True)
    k = torch.zeros((pages, page, kv, dim), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    scores = torch.zeros((pages, kv, page), device=DEV)
    positions = torch.zeros((pages, kv, page), dtype=torch.int32, device=DEV)
    far = pages - c.k.shape[0]
    for big, x in ((k, c.k), (v, c.v), (scores, c.scores), (positions, c.positions)):
        big[far:] = x.to(DEV)
    table = torch.where(c.table >= 0, c.table + far, c.table).to(DEV)
    cache = g10.CacheBuffers(k, v, table, c.lengths.to(DEV), scores=scores, positions=positions)
    q = queries(c, 1, 4, 6)
    r = O.attend(c, q, 0.1)
    out = g10.g10_cache_attend(cache, q.to(DEV), scale=0.1, add_scores=True)
    assert ((out.cpu().double() - r.out).abs() <= O.attend_bounds(c, r)[0]).all()
    c.scores = scores[far:].cpu()
    p = g10.g10_cache_plan_evictions(cache, 100, 2, 10)
    moves, lengths = O.plan(c, 100, 2, 10)
    check_plan(p, moves, lengths, c)
    g10.g10_cache_evict(cache, p.moves, p.counts)
    O.evict(c, moves)
    new = torch.randn(2, 1, kv, dim).to(torch.bfloat16)
    g10.g10_cache_append(cache, new.to(DEV), new.to(DEV))
    for s, n in enumerate(c.lengths.tolist()):
        pg, pl = O.places(c, s, n)
        c.k[pg[-1], pl[-1]] = c.v[pg[-1], pl[-1]] = new[s, 0]
    assert same(k[far:], c.k) and same(v[far:], c.v)
    assert int(cache.status.item()) == 0 and not k[:far].any() and not v[:far].any()


# ---- append ----------------------------------------------------------------------------------------------------------
def check_append(g10, c, new, group, rotary, interleaved, norm, counts=None, rows=4000, layout_q="side", seed=1):
    gen = torch.Generator().manual_seed(seed)
    heads, kv, dim = c.kv_heads * group, c.kv_heads, c.head_dim
    both = torch.randn(len(c.lengths), new, heads + 2 * kv, dim, generator=gen).to(c.dtype)
    q, k, v = both[:, :, :heads], both[:, :, heads:heads + kv], both[:, :, heads + kv:]
    qw, kw = ((1 + 0.3 * torch.randn(dim, generator=gen)).to(c.dtype) if norm else None for _ in range(2))
    cos = sin = None
    if rotary:
        angle = torch.rand(rows, rotary // 2, generator=gen, dtype=torch.float64) * 6.28
        cos, sin = angle.cos().float(), angle.sin().float()
    cache = O.upload(g10, c)
    on = lambda x: None if x is None else x.to(DEV)
    db = both.to(DEV)
    out = g10.g10_cache_append(cache, db[:, :, heads:heads + kv], db[:, :, heads + kv:], db[:, :, :heads] if group else None, q_weight=on(qw), k_weight=on(kw),
                               eps=1e-5, cos=on(cos), sin=on(sin), interleaved=interleaved, counts=on(counts))
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    seen = (c.seen if c.seen is not None else c.lengths).tolist()
    got_k, got_v = cache.k.cpu(), cache.v.cpu()
    want_scores = None if c.scores is None else c.scores.clone()
    want_positions = None if c.positions is None else c.positions.clone()
    # Norm and rotation in 32 bits: a mean of D squares, a reciprocal root, five products and a sum: (D + 16) * 2^-23 of the sizes that go in
    # (|x| + |partner|, normed), then one rounding.
    step, slip = O.half_step(c.dtype), (dim + 16) * 2.0 ** -23

    def near(got, x, w, position):
        want = O.turned(x, w, 1e-5, cos, sin, position, interleaved)
        size = O.turned(x.double().abs(), None if w is None else w.double().abs(), 1e-5, None, None, 0, False)
        if rotary:
            size = size + size[:rotary].max()
        bound = slip * size + step * (want.abs() + slip * size) + (2.0 ** -25 if c.dtype == torch.float16 else 0.0)
        return ((got.double() - want).abs() <= bound).all()

    owned = torch.zeros(c.k.shape[:2], dtype=torch.bool)
    for s, (length, count) in enumerate(zip(c.lengths.tolist(), O.counts_of(c, counts, new))):
        pg, pl = O.places(c, s, length)
        for t in range(count):
            slot, position = length - count + t, seen[s] - count + t
            a, b = int(pg[slot]), int(pl[slot])
            owned[a, b] = True
            for h in range(heads):
                assert near(out[s, t, h].cpu(), q[s, t, h], qw, position)
            for h in range(kv):
                assert near(got_k[a, b, h], k[s, t, h], kw, position)
                assert same(got_v[a, b, h], v[s, t, h])
                if want_scores is not None:
                    want_scores[a, h, b] = 0
                if want_positions is not None:
                    want_positions[a, h, b] = position
        if group:
            assert (out[s, count:] == 0).all()
    assert same(got_k[~owned], c.k[~owned]) and same(got_v[~owned], c.v[~owned])          # all else as it was
    if want_scores is not None:
        assert same(cache.scores, want_scores)
    if want_positions is not None:
        assert torch.equal(cache.positions.cpu(), want_positions)


@pytest.mark.parametrize("dim,rotary,interleaved", [(8, 8, False), (8, 4, True), (24, 10, False), (64, 64, False), (64, 32, True), (72, 72, False), (80, 40, False),
                                                    (80, 80, True), (96, 0, False), (128, 128, False), (128, 64, True), (192, 128, False), (256, 256, False),
                                                    (256, 2, False), (256, 2, True)])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_append_dims(g10, dim, rotary, interleaved, kind):
    c = O.make_cache([3, 17, 40, 1], 2, dim, 16, O.TYPES[kind], dim + rotary, positions=True)
    check_append(g10, c, 1, 3, rotary, interleaved, True)
    check_append(g10, c, 3, 1, rotary, interleaved, False, counts=torch.tensor([3, 0, 2, 3], dtype=torch.int32))


@pytest.mark.parametrize("page", [1, 5, 16, 64])
@pytest.mark.parametrize("layout", ["slots", "heads", "wide"])
@pytest.mark.parametrize("group", [0, 1, 5])
def test_append_pages_and_strides(g10, page, layout, group):
    c = O.make_cache([0, 1, 33, 64, 70], 3, 64, page, torch.bfloat16, page, layout=layout)
    c.seen = c.lengths + torch.tensor([0, 0, 1000, 5, 2000], dtype=torch.int32)
    check_append(g10, c, 4, group, 64, False, True)


def test_append_without_scores_and_many_tokens(g10):
    c = O.make_cache([700, 650], 2, 64, 16, torch.float16, 5, scores=False)
    check_append(g10, c, 640, 2, 32, True, True, counts=torch.tensor([640, 7], dtype=torch.int32))


# ---- plan and evict --------------------------------------------------------------------------------------------------
def check_plan(p, moves, lengths, c):
    got, counts = p.moves.cpu(), p.counts.cpu()
    assert p.new_lengths.tolist() == lengths
    for (s, h), pairs in moves.items():
        assert int(counts[s, h]) == len(pairs)
        assert got[s, h, :len(pairs)].tolist() == [list(x) for x in pairs]


def check_plan_and_evict(g10, c, budget, sinks, recent):
    cache = O.upload(g10, c)
    marked = torch.full((len(c.lengths), c.kv_heads, budget, 2), -5, dtype=torch.int32, device=DEV)
    p = g10.g10_cache_plan_evictions(cache, budget, sinks, recent, moves=marked)
    moves, lengths = O.plan(c, budget, sinks, recent)
    check_plan(p, moves, lengths, c)
    for (s, h), pairs in moves.items():
        assert (p.moves[s, h, len(pairs):] == -5).all()
    assert same(cache.scores, c.scores) and torch.equal(cache.lengths.cpu(), c.lengths)
    O.evict(c, moves)
    for _ in range(2):                                   # (a second time: the same)
        g10.g10_cache_evict(cache, p.moves, p.counts)
        assert same(cache.k, c.k) and same(cache.v, c.v) and same(cache.scores, c.scores)
        assert c.positions is None or torch.equal(cache.positions.cpu(), c.positions)
    assert int(cache.status.item()) == 0


def shuffle_positions(c, seed):
    rng = np.random.default_rng(seed)
    c.seen = c.lengths + 50
    for s, n in enumerate(c.lengths.tolist()):
        pg, pl = O.places(c, s, n)
        for h in range(c.kv_heads):
            c.positions[pg, h, pl] = torch.from_numpy(np.sort(rng.permutation(n + 50)[:n])[rng.permutation(n)].astype(np.int32))


@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (32, 4, 8), (100, 0, 100), (100, 100, 0), (257, 3, 50), (1000, 10, 10)])
@pytest.mark.parametrize("order", ["slots", "mixed"])
def test_plan_and_evict(g10, budget, sinks, recent, order):
    c = O.make_cache([0, 1, budget, budget + 1, budget + 2, 2 * budget + 7, 900], 2, 64, 16, torch.bfloat16, budget, positions=True)
    if order == "mixed":
        shuffle_positions(c, budget)
    check_plan_and_evict(g10, c, budget, sinks, recent)


@pytest.mark.parametrize("kind", ["equal", "few", "special", "zeros"])
def test_plan_with_ties_and_special_scores(g10, kind):
    c = O.make_cache([2500, 1300, 64], 3, 8, 32, torch.float16, 4, positions=True)
    rng = np.random.default_rng(1)
    n = c.scores.numel()
    values = {"equal": [1.5], "few": [0.0, 1.0, 2.0], "special": [math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -1e-45, 3.4e38, -1.0], "zeros": [0.0, -0.0]}[kind]
    c.scores = torch.from_numpy(rng.choice(np.array(values, dtype=np.float32), size=n)).view(c.scores.shape)
    check_plan_and_evict(g10, c, 700, 2, 3)


@pytest.mark.parametrize("page,layout", [(1, "slots"), (7, "heads"), (64, "wide"), (300, "slots")])
def test_evict_pages_and_strides(g10, page, layout):
    c = O.make_cache([400, 222], 2, 72, page, torch.bfloat16, page, layout=layout, positions=True)
    check_plan_and_evict(g10, c, 130, 1, 20)


@pytest.mark.parametrize("lengths,budget", [([70001], 4000), ([30000, 100, 45000], 128), ([5000] * 20, 4990), ([2111] * 40, 2048)])
def test_plan_long(g10, lengths, budget):
    c = O.make_cache(lengths, 2, 8, 64, torch.bfloat16, len(lengths), positions=True)
    shuffle_positions(c, 3)
    check_plan_and_evict(g10, c, budget, 4, budget // 8)


def test_plan_without_positions(g10):
    c = O.make_cache([500, 300], 2, 64, 16, torch.bfloat16, 3)
    check_plan_and_evict(g10, c, 200, 4, 30)


# ---- what is wrong in the data ---------------------------------------------------------------------------------------
def test_bad_pages_lengths_positions_and_moves_are_reported(g10):
    c = O.make_cache([40, 40], 2, 64, 16, torch.bfloat16, 3, positions=True)
    q, new = queries(c, 1, 2, 1).to(DEV), torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    before = c.k.clone(), c.v.clone()

    def calls(cache):
        p = g10.g10_cache_plan_evictions(cache, 20)
        g10.g10_cache_attend(cache, q, add_scores=True)
        g10.g10_cache_append(cache, new, new)
        return p

    for page in (-1, -2 ** 31, c.k.shape[0], 2 ** 31 - 1):
        c.table[1, 2] = page
        cache = O.upload(g10, c)
        p = calls(cache)
        g10.g10_cache_evict(cache, p.moves, p.counts)
        assert int(cache.status.item()) == 0x400
    c.table[1, 2] = c.table[1, 1]
    for length in (-1, -2 ** 31, 49, 2 ** 31 - 1):
        c.lengths[1] = length
        cache = O.upload(g10, c)
        calls(cache)
        assert int(cache.status.item()) & 0x800
    c.lengths[1] = 40
    for count in (-1, 2, 2 ** 31 - 1):
        cache = O.upload(g10, c)
        g10.g10_cache_attend(cache, q, counts=torch.tensor([1, count], dtype=torch.int32, device=DEV))
        assert int(cache.status.item()) == 0x800
        cache.status.zero_()
        g10.g10_cache_append(cache, new, new, counts=torch.tensor([count, 1], dtype=torch.int32, device=DEV))
        assert int(cache.status.item()) == 0x800
    for seen in (0, 31, 2 ** 31 - 1):                    # positions -1, 30, 2^31 - 2 in tables of 30 rows
        c.seen = torch.tensor([20, seen], dtype=torch.int32)
        cache = O.upload(g10, c)
        table = torch.ones(30, 32, device=DEV)
        g10.g10_cache_append(cache, new, new, cos=table, sin=table)
        assert int(cache.status.item()) == 0x1000
    cache = O.upload(g10, c)
    moves = torch.tensor([[19, 0], [40, 1], [-1, 2], [30, 20], [30, -1], [2 ** 31 - 1, 3]], dtype=torch.int32, device=DEV)
    plan = torch.zeros(2, 2, 20, 2, dtype=torch.int32, device=DEV)
    plan[:, :, :6] = moves
    for count in (6, -1, 21):
        cache.status.zero_()
        g10.g10_cache_evict(cache, plan, torch.full((2, 2), count, dtype=torch.int32, device=DEV))
        assert int(cache.status.item()) == 0x2000
    assert same(cache.k, before[0]) and same(cache.v, before[1])


# ---- as they are used ------------------------------------------------------------------------------------------------
def test_graphs_streams_and_workspaces(g10):
    """Two captured steps with a workspace each, replayed side by side after the lengths have moved on, beside eager calls on a third stream."""
    c = O.make_cache([700, 90, 1500], 2, 128, 16, torch.bfloat16, 12)
    q = queries(c, 1, 4, 1)
    dq = q.to(DEV)
    full = c.lengths.clone()
    cache = O.upload(g10, c)
    graphs = []
    for i in range(2):
        out, lse = torch.empty_like(dq), torch.empty(dq.shape[:3], device=DEV)
        ws = torch.empty(g10.g10_cache_workspace_bytes(cache, 1, 8), dtype=torch.uint8, device=DEV)
        g10.g10_cache_attend(cache, dq, out=out, lse=lse, ws=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            g10.g10_cache_attend(cache, dq, out=out, lse=lse, ws=ws)
        graphs.append((g, out, torch.cuda.Stream()))
    side = torch.cuda.Stream()
    for cut in (0, 64, 89):
        c.lengths = full - cut
        cache.lengths.copy_(c.lengths)
        torch.cuda.synchronize()
        r = O.attend(c, q, 128 ** -0.5)
        bound = O.attend_bounds(c, r)[0]
        for _ in range(20):
            for g, _, stream in graphs:
                with torch.cuda.stream(stream):
                    g.replay()
            eager = g10.g10_cache_attend(cache, dq, stream=side)
        torch.cuda.synchronize()
        for out in [eager] + [x[1] for x in graphs]:
            assert ((out.cpu().double() - r.out).abs() <= bound).all()
    cache.lengths.copy_(full)
    table = torch.ones(2000, 64, device=DEV)
    new = torch.randn(3, 1, 2, 128).to(torch.bfloat16).to(DEV)
    moves, counts, lengths = (torch.empty(s, dtype=torch.int32, device=DEV) for s in ((3, 2, 500, 2), (3, 2), (3,)))

    def step():
        g10.g10_cache_append(cache, new, new, dq, cos=table, sin=table, q_out=dq_out)
        g10.g10_cache_plan_evictions(cache, 500, 4, 100, moves=moves, counts=counts, new_lengths=lengths)
        g10.g10_cache_evict(cache, moves, counts)

    dq_out = torch.empty_like(dq)
    step()
    torch.cuda.synchronize()
    state = [x.clone() for x in (cache.k, cache.v, cache.scores)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    cache.scores.copy_(torch.rand_like(cache.scores))
    c.k, c.v, c.scores = cache.k.cpu(), cache.v.cpu(), cache.scores.cpu()
    g.replay()
    torch.cuda.synchronize()
    c.lengths = full
    for s, n in enumerate(full.tolist()):
        pg, pl = O.places(c, s, n)
        c.scores[pg[-1], :, pl[-1]] = 0
        c.k[pg[-1], pl[-1]], c.v[pg[-1], pl[-1]] = state[0].cpu()[pg[-1], pl[-1]], state[1].cpu()[pg[-1], pl[-1]]
    want, new_lengths = O.plan(c, 500, 4, 100)
    O.evict(c, want)
    assert lengths.tolist() == new_lengths
    assert same(cache.k, c.k) and same(cache.v, c.v) and same(cache.scores, c.scores)


@pytest.mark.parametrize("new,group", [(1, 4), (3, 4), (8, 7)])
def test_captured_booking(g10, new, group):
    """A captured call that books, replayed after the lengths have moved, three times in a row with nothing between."""
    c = O.make_cache([700, 90, 1500, 64], 2, 128, 16, torch.bfloat16, 21)
    q = queries(c, new, group, 3)
    cache, dq = O.upload(g10, c), q.to(DEV)
    out = torch.empty_like(dq)
    ws = torch.empty(g10.g10_cache_workspace_bytes(cache, new, 2 * group, add_scores=True), dtype=torch.uint8, device=DEV)
    g10.g10_cache_attend(cache, dq, out=out, ws=ws, add_scores=True)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        g10.g10_cache_attend(cache, dq, out=out, ws=ws, add_scores=True)
    c.lengths = c.lengths - 40
    cache.lengths.copy_(c.lengths)
    cache.scores.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    r = O.attend(c, q, 128 ** -0.5)
    bound, _, rel = O.attend_bounds(c, r)
    assert ((out.cpu().double() - r.out).abs() <= bound).all()
    got = cache.scores.cpu().double()
    for (s, h), w in r.booked.items():
        pg, pl = O.places(c, s, len(w))
        # (three additions to a score, each rounded)
        assert ((got[pg, h, pl] - 3 * w).abs() <= 3 * w * (float(rel[s].max()) * 1.01 + 2.0 ** -23) + 1e-30).all()


def test_what_a_call_allocates_on_another_stream_is_its_own(g10):
    """Memory that the current stream has given back may still have work ahead of it there: a call on another stream does not get it."""
    c = O.make_cache([300, 90], 2, 64, 16, torch.bfloat16, 5)
    q = queries(c, 1, 4, 5)
    cache, dq = O.upload(g10, c), q.to(DEV)
    side = torch.cuda.Stream()
    r = O.attend(c, q, 64 ** -0.5)
    bound = O.attend_bounds(c, r)[0]
    size = g10.g10_cache_workspace_bytes(cache, 1, 8)
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    for given in (dq.numel() * 2, size):
        x = torch.empty(given, dtype=torch.uint8, device=DEV)
        x.fill_(255)
        del x
    out = g10.g10_cache_attend(cache, dq, stream=side)
    torch.cuda.synchronize()
    assert ((out.cpu().double() - r.out).abs() <= bound).all()


@pytest.mark.parametrize("new", [1, 9])
def test_largest_windows(g10, new):
    most = 2 ** 31 - 1
    c = O.make_cache([300, 0, 65], 2, 64, 16, torch.float16, 8)
    q = queries(c, new, 4, 2)
    for window, sinks in ((most, 0), (most, most), (1, most), (70, most)):
        check_attend(g10, c, q, window=window, sinks=sinks, book=True)


def test_calls_of_two_threads(g10):
    import threading
    c = O.make_cache([900, 33, 400], 2, 128, 16, torch.bfloat16, 31)
    cases = [(1, 4), (8, 6)]
    wrong = []

    def work(new, group):
        with torch.cuda.device(0), torch.cuda.stream(torch.cuda.Stream()):
            q = queries(c, new, group, new)
            cache, dq = O.upload(g10, c), q.to(DEV)
            outs = [g10.g10_cache_attend(cache, dq) for _ in range(30)]
            torch.cuda.current_stream().synchronize()
            r = O.attend(c, q, 128 ** -0.5)
            bound = O.attend_bounds(c, r)[0]
            wrong.extend(1 for out in outs if not ((out.cpu().double() - r.out).abs() <= bound).all())
            wrong.extend(1 for _ in range(int(cache.status.item() != 0)))

    threads = [threading.Thread(target=work, args=x) for x in cases * 2]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_shared_rows_and_pages_of_sequences_that_attend(g10):
    """The same pages in two tables, and one query for all sequences, by a stride of zero."""
    c = O.make_cache([200, 200, 130], 2, 64, 16, torch.bfloat16, 17)
    c.table[1] = c.table[0]
    q = queries(c, 1, 4, 6)[:1].expand(3, -1, -1, -1)
    cache = O.upload(g10, c)
    out = g10.g10_cache_attend(cache, q[:1].to(DEV).expand(3, -1, -1, -1))
    r = O.attend(c, q, 64 ** -0.5)
    assert ((out.cpu().double() - r.out).abs() <= O.attend_bounds(c, r)[0]).all()


def test_binding_refusals(g10):
    c = O.make_cache([40, 20], 2, 64, 16, torch.bfloat16, 1, positions=True)
    cache = O.upload(g10, c)
    q = torch.zeros(2, 1, 8, 64, dtype=torch.bfloat16, device=DEV)
    kv = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    table = torch.zeros(50, 32, device=DEV)
    ints = torch.zeros(2, dtype=torch.int32, device=DEV)
    plan = g10.g10_cache_plan_evictions(cache, 8)
    state = [x.clone() for x in (cache.k, cache.v, cache.scores)]
    attend = [(q.float(), {}), (q.half(), {}), (q.cpu(), {}), (q[:1], {}), (q[..., :32], {}), (q[0], {}), (q.transpose(2, 3).contiguous().transpose(2, 3), {}),
              (q[:, :, :7], {}), (q, dict(out=q.float())), (q, dict(out=torch.empty(2, 1, 8, 128, dtype=q.dtype, device=DEV)[..., ::2])), (q, dict(lse=ints)),
              (q, dict(counts=ints.long())), (q, dict(counts=ints[:1])), (q, dict(ws=torch.empty(64, dtype=torch.uint8, device=DEV))), (q, dict(ws=ints)),
              (q, dict(window=5)), (q, dict(scale=math.inf)), (q[:, :0], {}), (torch.zeros(2, 300, 8, 64, dtype=q.dtype, device=DEV), {})]
    for x, kw in attend:
        with pytest.raises(g10.G10Error):
            g10.g10_cache_attend(cache, x, **kw)
    append = [((kv.float(), kv), {}), ((kv, kv.cpu()), {}), ((kv[:, :, :1], kv), {}), ((kv, kv.expand(2, 1, 2, 64)[:, :, :, :32]), {}), ((kv, kv), dict(cos=table)),
              ((kv, kv), dict(cos=table, sin=table[:, :16])), ((kv, kv), dict(cos=table.double(), sin=table.double())), ((kv, kv), dict(k_weight=table[0])),
              ((kv, kv), dict(q=q[:1])), ((kv, kv), dict(q=q, q_out=q[:, :, :4])), ((kv, kv), dict(counts=ints.long())),
              ((kv, kv), dict(cos=torch.zeros(9, 40, device=DEV), sin=torch.zeros(9, 40, device=DEV)))]
    for x, kw in append:
        with pytest.raises(g10.G10Error):
            g10.g10_cache_append(cache, *x, **kw)
    for moves, counts in [(plan.moves.long(), plan.counts), (plan.moves[:1], plan.counts), (plan.moves, plan.counts[:, :1]), (plan.moves.cpu(), plan.counts), (plan.moves[0], plan.counts)]:
        with pytest.raises(g10.G10Error):
            g10.g10_cache_evict(cache, moves, counts)
    for kw in (dict(budget=0), dict(budget=8, sinks=5, recent=4), dict(budget=8, counts=ints)):
        with pytest.raises(g10.G10Error):
            g10.g10_cache_plan_evictions(cache, **kw)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    assert all(same(a, b) for a, b in zip(state, (cache.k, cache.v, cache.scores)))


def test_a_conversation_within_a_budget(g10):
    """Prompts of different lengths, their last tokens looked at, eviction, then token after token with an eviction every few: two layers
    that share lengths.  Each step is compared with the definitions applied to the device's state before it."""
    budget, page, kv, group, dim, room = 48, 16, 2, 3, 64, 8
    prompts = [70, 12, 130]
    gen = torch.Generator().manual_seed(3)
    columns = -(-(max(prompts) + 40) // page)
    pages = columns * 3 + 2
    table = torch.randperm(pages, generator=gen)[:columns * 3].view(3, columns).int()
    lengths, seen = torch.tensor(prompts, dtype=torch.int32), torch.tensor(prompts, dtype=torch.int32)
    d_lengths, d_seen, d_table = lengths.to(DEV), seen.to(DEV), table.to(DEV)
    angle = torch.arange(400, dtype=torch.float64)[:, None] * torch.pow(10000.0, -torch.arange(dim // 2, dtype=torch.float64) / (dim // 2))[None]
    cos, sin = angle.cos().float().to(DEV), angle.sin().float().to(DEV)
    weight = torch.ones(dim, dtype=torch.bfloat16, device=DEV)
    layers = []
    for _ in range(2):
        k = torch.full((pages, page, kv, dim), math.nan, dtype=torch.bfloat16, device=DEV)
        cells = (pages, kv, page)
        layers.append(g10.CacheBuffers(k, k.clone(), d_table, d_lengths, seen=d_seen, scores=torch.full(cells, math.nan, device=DEV),
                                       positions=torch.full(cells, -1, dtype=torch.int32, device=DEV)))

    def host(cache):
        from types import SimpleNamespace
        return SimpleNamespace(k=cache.k.cpu(), v=cache.v.cpu(), table=table, lengths=d_lengths.cpu(), seen=d_seen.cpu(), page_size=page, kv_heads=kv, head_dim=dim,
                               dtype=torch.bfloat16, scores=cache.scores.cpu(), positions=cache.positions.cpu())

    def turn(new, counts):
        for cache in layers:
            both = torch.randn(3, new, kv * (group + 2), dim, generator=gen).to(torch.bfloat16).to(DEV)
            q = g10.g10_cache_append(cache, both[:, :, kv * group:kv * (group + 1)], both[:, :, kv * (group + 1):], both[:, :, :kv * group], q_weight=weight,
                                     k_weight=weight, cos=cos, sin=sin, counts=counts.to(DEV))
            last = int(min(new, 8))
            # (the last tokens of each sequence look at the whole cache)
            at = (counts[:, None] - torch.minimum(counts, torch.tensor(last))[:, None] + torch.arange(last)[None]).clamp(max=new - 1).long().to(DEV)
            looks = torch.minimum(counts, torch.tensor(last)).int()
            q = q.gather(1, at[:, :, None, None].expand(-1, -1, kv * group, dim)).contiguous()
            c = host(cache)
            r = O.attend(c, q.cpu(), dim ** -0.5, counts=looks)
            b_out, _, rel = O.attend_bounds(c, r)
            out = g10.g10_cache_attend(cache, q, counts=looks.to(DEV), add_scores=True).cpu().double()
            assert ((out - r.out).abs() <= b_out).all()
            after = cache.scores.cpu()
            for (s, h), w in r.booked.items():
                pg, pl = O.places(c, s, len(w))
                was = c.scores[pg, h, pl].double()
                assert ((after[pg, h, pl].double() - was - w).abs() <= w * float(rel[s].max()) + 2.0 ** -23 * (was + w)).all()

    def evict():
        for cache in layers:
            c = host(cache)
            p = g10.g10_cache_plan_evictions(cache, budget, 2, 8)
            moves, planned = O.plan(c, budget, 2, 8)
            check_plan(p, moves, planned, c)
            g10.g10_cache_evict(cache, p.moves, p.counts)
            O.evict(c, moves)
            assert same(cache.k, c.k) and same(cache.v, c.v) and same(cache.scores, c.scores) and torch.equal(cache.positions.cpu(), c.positions)
        d_lengths.copy_(p.new_lengths)

    turn(max(prompts), torch.tensor(prompts, dtype=torch.int32))
    evict()
    for i in range(2 * room):
        d_lengths.add_(1)
        d_seen.add_(1)
        turn(1, torch.ones(3, dtype=torch.int32))
        if i % room == room - 1:
            evict()
    assert d_lengths.tolist() == [budget, 28, budget] and d_seen.tolist() == [n + 2 * room for n in prompts]
    for cache in layers:
        assert int(cache.status.item()) == 0
        c = host(cache)
        for s, n in enumerate(c.lengths.tolist()):       # first and last tokens are all there
            pg, pl = O.places(c, s, n)
            for h in range(kv):
                have = set(c.positions[pg, h, pl].tolist())
                assert len(have) == n and {0, 1} <= have and set(range(prompts[s] + 2 * room - 8, prompts[s] + 2 * room)) <= have
