"""The key-value cache of 8-bit rows on the device against the definitions in 64 bits (packed_oracle.py)."""
import math

import numpy as np
import pytest
import torch

import cache_oracle as O
import packed_oracle as P

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
    kind = {1: torch.int8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.contiguous().view(kind).cpu(), b.contiguous().view(kind).cpu())


def queries(c, new, group, seed, spread=2.0):
    gen = torch.Generator().manual_seed(seed + 77)
    return (spread * torch.randn(len(c.lengths), new, c.kv_heads * group, c.head_dim, generator=gen)).to(c.dtype)


def reference(c, q, window=0, sinks=0, counts=None, scale=None):
    """What the call gives, and how far it may be off."""
    scale = c.head_dim ** -0.5 if scale is None else scale
    P.values(c)
    r = O.attend(c, q, scale, window, sinks, counts)
    return (r,) + P.attend_bounds(c, r, q, scale)


def check_attend(g10, c, q, window=0, sinks=0, counts=None, book=False, scale=None, strided=False):
    cache = P.upload(g10, c)
    dq = q.to(DEV)
    if strided:
        wide = torch.full(q.shape[:2] + (q.shape[2] + 3, q.shape[3]), math.nan, dtype=q.dtype, device=DEV)
        wide[:, :, 1:-2] = dq
        dq = wide[:, :, 1:-2]
    lse = torch.full(q.shape[:3], 99.0, device=DEV)
    out = torch.full(q.shape, 99.0, dtype=q.dtype, device=DEV)
    dc = None if counts is None else counts.to(DEV)
    g10.g10_packed_attend(cache, dq, scale=scale, window=window, sinks=sinks, counts=dc, add_scores=book, out=out, lse=lse)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    r, b_out, b_lse, rel = reference(c, q, window, sinks, counts, scale)
    out, lse = out.cpu().double(), lse.cpu().double()
    nothing = torch.isinf(r.lse)
    assert torch.isfinite(out).all()
    assert (out[nothing] == 0).all()
    off = (out - r.out).abs() - b_out
    assert off.max() <= 0, "out off by %g over the bound at %s" % (off.max(), np.unravel_index(int(off.argmax()), off.shape))
    assert torch.equal(torch.isinf(lse), nothing)
    assert ((lse - r.lse).abs() <= b_lse)[~nothing].all()
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


both = pytest.mark.parametrize("code", ["int8", "e4m3"])


# ---- attend ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dim", [16, 32, 48, 64, 80, 96, 112, 128, 144, 192, 208, 256])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@both
def test_attend_head_dims(g10, dim, kind, code):
    c = P.make_packed([0, 1, 63, 64, 65, 200], 2, dim, 16, O.TYPES[kind], code, dim)
    check_attend(g10, c, queries(c, 1, 4, dim), book=True)
    check_attend(g10, c, queries(c, 3, 4, dim), book=True)
    check_attend(g10, c, queries(c, 9, 4, dim), book=True)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 15, 16, 17, 40])
@pytest.mark.parametrize("book", [False, True])
@both
def test_attend_groups(g10, group, book, code):
    c = P.make_packed([7, 129, 300, 0, 31], 3, 64, 8, torch.bfloat16, code, group)
    check_attend(g10, c, queries(c, 1, group, group), book=book, strided=book)


@pytest.mark.parametrize("page", [1, 3, 7, 16, 48, 64, 100, 256])
@pytest.mark.parametrize("layout", ["slots", "heads", "wide"])
@both
def test_attend_pages_and_strides(g10, page, layout, code):
    c = P.make_packed([1, 5, 97, 100, 101, 333], 2, 128, page, torch.float16, code, page, layout=layout)
    check_attend(g10, c, queries(c, 1, 4, page), book=True)


@pytest.mark.parametrize("new,group", [(2, 1), (3, 4), (5, 3), (16, 1), (2, 8), (16, 4), (33, 2), (16, 16), (130, 3)])
@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("fp16", 80)])
@both
def test_attend_several_tokens(g10, new, group, kind, dim, code):
    lengths = [new + 61, new, 1, 0, new + 200, max(1, new // 2)]
    c = P.make_packed(lengths, 2, dim, 16, O.TYPES[kind], code, new * group)
    check_attend(g10, c, queries(c, new, group, new), book=True)
    counts = torch.tensor([new, max(1, new // 3), 1, 0, 0, new], dtype=torch.int32)
    check_attend(g10, c, queries(c, new, group, new + 1), book=True, counts=counts)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 5), (64, 64), (65, 1), (100, 70), (5000, 5000), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("new,group", [(1, 4), (6, 1), (40, 2)])
@both
def test_attend_window_and_sinks(g10, window, sinks, new, group, code):
    c = P.make_packed([1, 64, 130, 400, 777, 0], 2, 64, 24, torch.bfloat16, code, min(window, 99))
    check_attend(g10, c, queries(c, new, group, sinks), window=window, sinks=sinks, book=True)


@pytest.mark.parametrize("dim", [16, 80, 128, 192, 256])
@pytest.mark.parametrize("group,new", [(1, 1), (4, 1), (7, 2), (3, 30)])
@both
def test_attend_with_room_in_the_table(g10, dim, group, new, code):
    lengths = [new + 1, new + 700, 0, 1, new + 64, 330]
    for page, columns in ((16, 400), (64, 1000)):
        c = P.make_packed(lengths, 2, dim, page, torch.bfloat16, code, dim + group, columns=columns)
        check_attend(g10, c, queries(c, new, group, dim), book=True)
        check_attend(g10, c, queries(c, new, group, dim + 1), window=150, sinks=70)


@pytest.mark.parametrize("tiles", [1, 2, 5, 8, 16, 31, 33])
@pytest.mark.parametrize("group", [1, 12])
@both
def test_attend_lengths_about_what_a_cluster_takes(g10, tiles, group, code):
    for lengths in ([64 * tiles], [64 * tiles - 63, 0, 1], [64 * tiles, 64, 65, 64 * tiles - 1]):
        c = P.make_packed(lengths, 2, 128, 32, torch.float16, code, tiles)
        check_attend(g10, c, queries(c, 1, group, tiles), book=True)
        check_attend(g10, c, queries(c, 1, group, tiles), window=100, sinks=3)


@pytest.mark.parametrize("lengths,kv,group,dim", [([9001], 1, 8, 128), ([20000, 3, 4000, 0, 900], 2, 4, 64), ([2500] * 7, 8, 16, 128), ([3000, 1], 1, 1, 256), ([5000] * 40, 4, 1, 64),
                                                  ([9001, 300], 2, 40, 128), ([4000] * 30, 2, 20, 80)])
@both
def test_attend_long(g10, lengths, kv, group, dim, code):
    c = P.make_packed(lengths, kv, dim, 64, torch.bfloat16, code, kv)
    check_attend(g10, c, queries(c, 1, group, 3), book=True)


@pytest.mark.parametrize("new", [1, 9])
@both
def test_attend_scales_far_apart(g10, new, code):
    """Values of any size beside one another, keys of none; queries of any size."""
    c = P.make_packed([300, 65, 700], 2, 64, 16, torch.bfloat16, code, 4)
    gen = torch.Generator().manual_seed(1)
    c.scales[..., 1] = torch.exp2(torch.randint(-90, 90, c.scales.shape[:3], generator=gen).float())
    P.values(c)
    check_attend(g10, c, queries(c, new, 4, 1))
    c.scales[..., 1] = 0.0
    c.scales[..., 0] = 0.0
    check_attend(g10, c, queries(c, new, 4, 1), book=True)
    for size in (2.0 ** -100, 2.0 ** 60):
        c = P.make_packed([300, 65, 700], 2, 64, 16, torch.bfloat16, code, 4)
        q = queries(c, new + 1, 4, 1)
        q *= size
        q[:, 0, ::2] *= 2.0 ** -30                       # (rows of their own sizes)
        check_attend(g10, c, q, scale=0.125 / size)
    c = P.make_packed([300, 65, 700], 2, 64, 16, torch.float16, code, 4)
    check_attend(g10, c, queries(c, new, 4, 1, spread=40.0))
    check_attend(g10, c, queries(c, new, 4, 1), scale=-0.3, book=True)


@pytest.mark.parametrize("new,group", [(1, 8), (3, 5), (30, 4)])
@both
def test_attend_where_later_slots_outweigh_all_before(g10, new, group, code):
    c = P.make_packed([1500], 1, 64, 16, torch.float16, code, 2, spread=0.0)
    pg, pl = O.places(c, 0, 1500)
    q = queries(c, new, group, 4)
    q[0] = q[0, :1, :1]
    # keys along the queries, longer and longer
    kc, scale = P.packed(q[0, 0, 0].double()[None] * torch.linspace(0.0, 3.0, 1500, dtype=torch.float64)[:, None], code)
    c.kc.view(torch.int8)[pg, pl, 0] = kc.view(torch.int8)
    c.scales[pg, 0, pl, 0] = scale
    check_attend(g10, c, q, book=True)


@pytest.mark.parametrize("new", [2, 5, 20])
@both
def test_attend_rows_that_are_no_numbers(g10, new, code):
    """A row of NaN makes what sees it NaN, and nothing else."""
    c = P.make_packed([130, 70], 2, 64, 16, torch.bfloat16, code, 9)
    q = queries(c, new, 2, 1)
    r, bound = reference(c, q)[:2]
    pg, pl = O.places(c, 0, 130)
    for side in (0, 1):
        cache = P.upload(g10, c)
        cache.scales[pg[129], 1, pl[129], side] = math.nan
        if code == "e4m3" and side == 1:                 # a code that is no number, by itself
            cache.scales[pg[129], 1, pl[129], side] = c.scales[pg[129], 1, pl[129], side] = 1.0
            cache.v.view(torch.int8)[pg[129], pl[129], 1, 3] = 127
            r, bound = reference(c, q)[:2]               # (its element aside, the row counts by that scale)
        lse = torch.empty(q.shape[:3], device=DEV)
        out = g10.g10_packed_attend(cache, q.to(DEV), lse=lse).cpu().double()
        bad = torch.zeros(q.shape, dtype=torch.bool)
        bad[0, new - 1, 2:, 3 if code == "e4m3" and side == 1 else slice(None)] = True
        assert torch.equal(torch.isnan(out), bad)
        assert ((out - r.out).abs() <= bound)[~bad].all()
        assert torch.isnan(lse).any() == (side == 0)


def test_offsets_beyond_32_bits(g10):
    """Rows more than 2^32 bytes into the pool."""
    page, kv, dim = 64, 8, 128
    pages = (1 << 32) // (page * kv * dim) + 40
    c = P.make_packed([200, 64], kv, dim, page, torch.bfloat16, "int8", 3)
    pool = [torch.empty(pages, page, kv, dim, dtype=torch.int8, device=DEV) for _ in range(2)]
    scales = torch.full((pages, kv, page, 2), math.nan, device=DEV)
    shift = pages - c.kc.shape[0]
    for to, x in ((pool[0], c.kc), (pool[1], c.vc), (scales, c.scales)):
        to[shift:] = x.to(DEV)
    table = torch.where(c.table >= 0, c.table + shift, c.table)
    cache = g10.PackedBuffers(*pool, scales, table.to(DEV), c.lengths.to(DEV))
    q = queries(c, 1, 4, 1)
    r, bound = reference(c, q)[:2]
    out = g10.g10_packed_attend(cache, q.to(DEV))
    k, v = g10.g10_packed_read(cache, 64)
    g10.g10_packed_append(cache, v[:, :1], v[:, 1:2])
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    assert ((out.cpu().double() - r.out).abs() <= bound).all()
    pg, pl = O.places(c, 0, 64)
    assert same(k[0], c.k[pg, pl].float().to(torch.bfloat16)) and same(v[0], c.v[pg, pl].float().to(torch.bfloat16))
    pg, pl = O.places(c, 0, 200)
    want = P.packed(v[0, 1].cpu().double(), "int8")[0]
    assert (pool[1][shift + pg[199], pl[199]].cpu().int() - want.int()).abs().max() <= 1


def test_attend_same_bits_each_time(g10):
    c = P.make_packed([9001, 300, 4000], 2, 128, 16, torch.bfloat16, "int8", 7)
    cache, dq = P.upload(g10, c), queries(c, 2, 4, 1).to(DEV)
    cache.scores.zero_()
    first = g10.g10_packed_attend(cache, dq, add_scores=True)
    booked = cache.scores.clone()
    for _ in range(5):
        cache.scores.zero_()
        assert same(g10.g10_packed_attend(cache, dq, add_scores=True), first) and same(cache.scores, booked)


# ---- append ----------------------------------------------------------------------------------------------------------
def check_append(g10, c, new, group, rotary, interleaved, norm, counts=None, rows=4000, seed=1, spoil=None):
    gen = torch.Generator().manual_seed(seed)
    heads, kv, dim = c.kv_heads * group, c.kv_heads, c.head_dim
    rows_of = torch.randn(len(c.lengths), new, heads + 2 * kv, dim, generator=gen).to(c.dtype)
    if spoil:
        spoil(rows_of[:, :, heads:])
    q, k, v = rows_of[:, :, :heads], rows_of[:, :, heads:heads + kv], rows_of[:, :, heads + kv:]
    qw, kw = ((1 + 0.3 * torch.randn(dim, generator=gen)).to(c.dtype) if norm else None for _ in range(2))
    cos = sin = None
    if rotary:
        angle = torch.rand(rows, rotary // 2, generator=gen, dtype=torch.float64) * 6.28
        cos, sin = angle.cos().float(), angle.sin().float()
    cache = P.upload(g10, c)
    on = lambda x: None if x is None else x.to(DEV)
    db = rows_of.to(DEV)
    out = g10.g10_packed_append(cache, db[:, :, heads:heads + kv], db[:, :, heads + kv:], db[:, :, :heads] if group else None, q_weight=on(qw), k_weight=on(kw),
                                eps=1e-5, cos=on(cos), sin=on(sin), interleaved=interleaved, counts=on(counts))
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    if group:                                            # queries: as into the other cache
        plain = O.make_cache(c.lengths.tolist(), kv, dim, c.page_size, c.dtype, 1)
        plain.seen = c.seen
        other = O.upload(g10, plain)
        assert same(out, g10.g10_cache_append(other, db[:, :, heads:heads + kv], db[:, :, heads + kv:], db[:, :, :heads], q_weight=on(qw), k_weight=on(kw),
                                              eps=1e-5, cos=on(cos), sin=on(sin), interleaved=interleaved, counts=on(counts)))
    seen = (c.seen if c.seen is not None else c.lengths).tolist()
    got = [x.cpu() for x in (cache.k, cache.v)]
    scales = cache.scales.cpu()
    want_scores, want_positions = (None if x is None else x.clone() for x in (c.scores, c.positions))
    slip = (dim + 16) * 2.0 ** -23                       # (norm and rotation in 32 bits: test_gpu_cache.py)
    owned = torch.zeros(c.kc.shape[:2], dtype=torch.bool)
    for s, (length, count) in enumerate(zip(c.lengths.tolist(), O.counts_of(c, counts, new))):
        pg, pl = O.places(c, s, length)
        for t in range(count):
            slot, position = length - count + t, seen[s] - count + t
            a, b = int(pg[slot]), int(pl[slot])
            owned[a, b] = True
            for h in range(kv):
                for side, x in ((0, k[s, t, h]), (1, v[s, t, h])):
                    want, error = x.double(), torch.zeros(dim, dtype=torch.float64)
                    if side == 0:
                        want = O.turned(x, kw, 1e-5, cos, sin, position, interleaved)
                        error = O.turned(x.double().abs(), None if kw is None else kw.double().abs(), 1e-5, None, None, 0, False)
                        error = slip * (error + (error[:rotary].max() if rotary else 0.0)) if norm or rotary else 0.0 * error
                    top, scale = want.abs().max(), float(scales[a, h, b, side])
                    codes = got[side][a, b, h].double()
                    if not torch.isfinite(want).all():
                        assert math.isnan(scale) and (codes == 0).all()
                    elif top < 2.0 ** -101:
                        assert scale == 0 and (codes == 0).all()
                    else:
                        # the scale: the largest element's error, and a division; a code: half a step (of the binade above, at its border), the error of what it stands
                        # for and three roundings of numbers up to Q
                        q_max = P.LARGEST[c.code]
                        assert abs(scale * q_max - top) <= error.max() + 2.0 ** -22 * top
                        in_units = want * q_max / top
                        off = error * q_max / top + q_max * (float(error.max() / top) + 2.0 ** -22)
                        assert ((codes - in_units).abs() <= P.step_of(in_units.abs() + off, c.code) / 2 + off).all()
                        assert codes.abs().max() == q_max
                if want_scores is not None:
                    want_scores[a, h, b] = 0
                if want_positions is not None:
                    want_positions[a, h, b] = position
    for side, x in ((0, c.kc), (1, c.vc)):               # all else as it was
        assert same(got[side].view(torch.int8)[~owned], x.view(torch.int8)[~owned])
    assert same(scales.transpose(1, 2)[~owned], c.scales.transpose(1, 2)[~owned])
    if want_scores is not None:
        assert same(cache.scores, want_scores)
    if want_positions is not None:
        assert torch.equal(cache.positions.cpu(), want_positions)


@pytest.mark.parametrize("dim,rotary,interleaved", [(16, 16, False), (16, 6, True), (48, 10, False), (64, 64, False), (64, 32, True), (80, 40, False), (80, 80, True),
                                                    (96, 0, False), (128, 128, False), (192, 128, False), (256, 256, False), (256, 2, True)])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@both
def test_append_dims(g10, dim, rotary, interleaved, kind, code):
    c = P.make_packed([3, 17, 40, 1], 2, dim, 16, O.TYPES[kind], code, dim + rotary, positions=True)
    check_append(g10, c, 1, 3, rotary, interleaved, True)
    check_append(g10, c, 3, 1, rotary, interleaved, False, counts=torch.tensor([3, 0, 2, 3], dtype=torch.int32))


@pytest.mark.parametrize("page", [1, 5, 64])
@pytest.mark.parametrize("layout", ["slots", "heads", "wide"])
@pytest.mark.parametrize("group", [0, 5])
@both
def test_append_pages_and_strides(g10, page, layout, group, code):
    c = P.make_packed([0, 1, 33, 64, 70], 3, 64, page, torch.bfloat16, code, page, layout=layout)
    c.seen = c.lengths + torch.tensor([0, 0, 1000, 5, 2000], dtype=torch.int32)
    check_append(g10, c, 4, group, 64, False, True)


@both
def test_append_many_tokens_without_scores(g10, code):
    c = P.make_packed([900, 0, 333], 2, 64, 16, torch.float16, code, 1, scores=False)
    check_append(g10, c, 300, 2, 32, True, True)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@both
def test_append_rows_of_any_size(g10, kind, code):
    """Zeros, infinities, NaN, rows of the smallest and of the largest numbers."""
    c = P.make_packed([12, 20], 2, 64, 8, O.TYPES[kind], code, 2)

    def spoil(x):                                        # [seqs, new, 2 kv, dim]
        top = torch.finfo(x.dtype).max
        x[0, 0] = 0
        x[0, 1, :, 5] = math.inf
        x[0, 2, :, 63] = math.nan
        x[0, 3, :, 0] = -math.inf
        x[0, 4] = x[0, 4].sign() * top
        x[0, 5] *= torch.finfo(x.dtype).tiny
        x[0, 6] = 0
        x[0, 6, :, 17] = torch.finfo(x.dtype).smallest_normal
        x[1, 0] = 1
        x[1, 1] *= 2.0 ** -20
    check_append(g10, c, 8, 1, 0, False, False, spoil=spoil)


# ---- read ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("page,layout", [(1, "slots"), (7, "heads"), (16, "wide"), (64, "slots")])
@pytest.mark.parametrize("kind,dim", [("bf16", 128), ("fp16", 80), ("bf16", 16), ("fp16", 256)])
@both
def test_read(g10, page, layout, kind, dim, code):
    c = P.make_packed([0, 1, 33, 64, 150], 3, dim, page, O.TYPES[kind], code, page, layout=layout)
    cache = P.upload(g10, c)
    for tokens, starts in ((1, None), (5, [0, 0, 30, 63, 149]), (160, None), (70, [-3, 2 ** 31 - 1, -2 ** 31, 60, 100]), (0, None)):
        starts_of = [0] * 5 if starts is None else starts
        ds = None if starts is None else torch.tensor(starts, dtype=torch.int32, device=DEV)
        k, v = g10.g10_packed_read(cache, tokens, starts=ds)
        # into parts of larger tensors, heads before tokens
        wide = torch.full((2, 5, 3, tokens + 2, dim + 8), 7.0, dtype=c.dtype, device=DEV)
        into = [wide[i, :, :, 1:tokens + 1, 8:].transpose(1, 2) for i in range(2)]
        assert g10.g10_packed_read(cache, tokens, starts=ds, k=into[0], v=into[1])[0] is into[0]
        only = torch.empty_like(v)
        g10.g10_packed_read(cache, tokens, starts=ds, v=only)
        want = torch.zeros(2, 5, tokens, 3, dim, dtype=c.dtype)
        for s, n in enumerate(c.lengths.tolist()):
            pg, pl = O.places(c, s, n)
            for t in range(tokens):
                slot = starts_of[s] + t
                if 0 <= slot < n:
                    for side, x in ((0, c.kc), (1, c.vc)):
                        want[side, s, t] = (x[pg[slot], pl[slot]].float() * c.scales[pg[slot], :, pl[slot], side, None]).to(c.dtype)
        torch.cuda.synchronize()
        assert int(cache.status.item()) == 0
        assert same(k, want[0]) and same(v, want[1]) and same(into[0], want[0]) and same(into[1], want[1]) and same(only, want[1])
        wide[:, :, :, 1:tokens + 1, 8:] = 7.0
        assert (wide == 7.0).all()


def test_read_of_what_is_no_number(g10):
    c = P.make_packed([9], 2, 64, 4, torch.bfloat16, "int8", 1)
    pg, pl = O.places(c, 0, 9)
    c.scales[pg[3], 1, pl[3], 0] = math.nan
    k, v = g10.g10_packed_read(P.upload(g10, c), 9)
    assert torch.isnan(k[0, 3, 1]).all() and torch.isnan(k).sum() == 64 and not torch.isnan(v).any()


def test_read_long(g10):
    c = P.make_packed([5000, 1, 4097], 2, 128, 16, torch.bfloat16, "e4m3", 1)
    k, v = g10.g10_packed_read(P.upload(g10, c), 5000)
    for s, n in enumerate(c.lengths.tolist()):
        pg, pl = O.places(c, s, n)
        for side, got, x in ((0, k, c.kc), (1, v, c.vc)):
            assert same(got[s, :n], (x[pg, pl].float() * c.scales[pg, :, pl, side, None]).to(c.dtype))
            assert (got[s, n:] == 0).all()


# ---- evict -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (32, 4, 8), (100, 0, 100), (257, 3, 50), (1000, 10, 10)])
@pytest.mark.parametrize("dim,page,layout", [(128, 16, "slots"), (16, 1, "heads"), (208, 7, "wide")])
@both
def test_plan_and_evict(g10, budget, sinks, recent, dim, page, layout, code):
    c = P.make_packed([0, 1, 99, 100, 101, 300, 555], 2, dim, page, torch.bfloat16, code, budget, positions=True, layout=layout)
    cache = P.upload(g10, c)
    p = g10.g10_cache_plan_evictions(cache, budget, sinks, recent)
    moves, lengths = O.plan(c, budget, sinks, recent)
    assert p.new_lengths.tolist() == lengths
    for (s, h), pairs in moves.items():
        n = int(p.counts[s, h])
        assert sorted(map(tuple, p.moves[s, h, :n].tolist())) == sorted(pairs)
    g10.g10_packed_evict(cache, p.moves, p.counts)
    P.evict(c, moves)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    assert same(cache.k, c.kc) and same(cache.v, c.vc) and same(cache.scales, c.scales) and same(cache.scores, c.scores) and torch.equal(cache.positions.cpu(), c.positions)


# ---- what the data may have wrong ------------------------------------------------------------------------------------
def test_bad_pages_lengths_and_moves_are_reported(g10):
    c = P.make_packed([20, 40], 2, 64, 8, torch.bfloat16, "int8", 6, columns=6, positions=True)
    before = [x.clone() for x in (c.kc, c.vc, c.scales)]
    q = queries(c, 1, 4, 1).to(DEV)
    new = torch.randn(2, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    for page in (-1, -2 ** 31, c.kc.shape[0], 2 ** 31 - 1):
        c.table[1, 4] = page
        cache = P.upload(g10, c)
        g10.g10_packed_attend(cache, q, add_scores=True)
        assert int(cache.status.item()) == 0x400
        cache.status.zero_()
        k, _ = g10.g10_packed_read(cache, 40)
        assert int(cache.status.item()) == 0x400 and (k[1, 32:] == 0).all() and (k[1, :32] != 0).any()
        cache.status.zero_()
        g10.g10_packed_append(cache, new, new)
        assert int(cache.status.item()) == 0x400
    c.table[1, 4] = c.table[1, 3]
    for length in (-1, -2 ** 31, 49, 2 ** 31 - 1):
        c.lengths[1] = length
        cache = P.upload(g10, c)
        g10.g10_packed_attend(cache, q)
        assert int(cache.status.item()) & 0x800
        cache.status.zero_()
        g10.g10_packed_read(cache, 4)
        assert int(cache.status.item()) & 0x800
    c.lengths[1] = 40
    cache = P.upload(g10, c)
    moves = torch.tensor([[19, 0], [40, 1], [-1, 2], [30, 20], [30, -1], [2 ** 31 - 1, 3]], dtype=torch.int32, device=DEV)
    plan = torch.zeros(2, 2, 20, 2, dtype=torch.int32, device=DEV)
    plan[:, :, :6] = moves
    for count in (6, -1, 21):
        cache.status.zero_()
        g10.g10_packed_evict(cache, plan, torch.full((2, 2), count, dtype=torch.int32, device=DEV))
        assert int(cache.status.item()) == 0x2000
    assert same(cache.k, before[0]) and same(cache.v, before[1]) and same(cache.scales, before[2])


def test_binding_refusals(g10):
    c = P.make_packed([40, 20], 2, 64, 16, torch.bfloat16, "int8", 1, positions=True)
    cache = P.upload(g10, c)
    plain = O.upload(g10, O.make_cache([40, 20], 2, 64, 16, torch.bfloat16, 1))
    q = torch.zeros(2, 1, 8, 64, dtype=torch.bfloat16, device=DEV)
    kv = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    ints = torch.zeros(2, dtype=torch.int32, device=DEV)
    plan = g10.g10_cache_plan_evictions(cache, 8)
    k, v, scales, table, lengths = cache.k, cache.v, cache.scales, cache.page_table, cache.lengths
    refused = [lambda: g10.g10_cache_attend(cache, q), lambda: g10.g10_cache_append(cache, kv, kv), lambda: g10.g10_cache_evict(cache, plan.moves, plan.counts),
               lambda: g10.g10_packed_attend(plain, q), lambda: g10.g10_packed_append(plain, kv, kv), lambda: g10.g10_packed_evict(plain, plan.moves, plan.counts),
               lambda: g10.g10_packed_read(plain, 4), lambda: g10.g10_cache_workspace_bytes(cache, 1, 8), lambda: g10.g10_packed_workspace_bytes(plain, 1, 8),
               lambda: g10.PackedBuffers(k, None, scales, table, lengths), lambda: g10.PackedBuffers(k.float(), v.float(), scales, table, lengths),
               lambda: g10.PackedBuffers(k, v, scales[..., 0], table, lengths), lambda: g10.PackedBuffers(k, v, scales.double(), table, lengths),
               lambda: g10.PackedBuffers(k, v, scales.cpu(), table, lengths), lambda: g10.PackedBuffers(k, v, scales, table, lengths, dtype=torch.float32),
               lambda: g10.PackedBuffers(k, v.view(torch.float8_e4m3fn), scales, table, lengths), lambda: setattr(cache, "scales", scales.clone()),
               lambda: g10.g10_packed_attend(cache, q.half()), lambda: g10.g10_packed_attend(cache, q[:, :, :7]), lambda: g10.g10_packed_attend(cache, q, window=5),
               lambda: g10.g10_packed_attend(cache, q, ws=torch.empty(64, dtype=torch.uint8, device=DEV)), lambda: g10.g10_packed_attend(cache, q, scale=math.nan),
               lambda: g10.g10_packed_append(cache, kv.half(), kv), lambda: g10.g10_packed_read(cache, -1), lambda: g10.g10_packed_read(cache, 2 ** 31),
               lambda: g10.g10_packed_read(cache, 1, starts=ints.long()), lambda: g10.g10_packed_read(cache, 2, k=kv), lambda: g10.g10_packed_read(cache, 1, k=kv.half()),
               lambda: g10.g10_packed_read(cache, 1, v=torch.zeros(2, 1, 2, 68, dtype=kv.dtype, device=DEV)[..., 4:]),
               lambda: g10.g10_packed_evict(cache, plan.moves.long(), plan.counts)]
    state = [x.clone() for x in (k, v, scales, cache.scores)]
    for call in refused:
        with pytest.raises(g10.G10Error):
            call()
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0 and all(same(a, b) for a, b in zip(state, (k, v, scales, cache.scores)))


# ---- as they are used ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("new,group", [(1, 4), (3, 4), (8, 7)])
@both
def test_captured_steps(g10, new, group, code):
    """A captured run of append, attend with booking, plan, evict and read, replayed twice beside eager calls on another stream, after the contents have moved on."""
    c = P.make_packed([700, 90, 1500, 64], 2, 128, 16, torch.bfloat16, code, 21)
    cache, other = P.upload(g10, c), P.upload(g10, c)
    heads = 2 * group
    gen = torch.Generator().manual_seed(4)
    x = torch.randn(4, new, heads + 4, 128, generator=gen).to(torch.bfloat16).to(DEV)
    ws = torch.empty(g10.g10_packed_workspace_bytes(cache, new, heads, add_scores=True), dtype=torch.uint8, device=DEV)
    out = torch.empty(4, new, heads, 128, dtype=torch.bfloat16, device=DEV)

    def step(cache, out, ws, stream=None):
        g10.g10_packed_append(cache, x[:, :, heads:heads + 2], x[:, :, heads + 2:], stream=stream)
        g10.g10_packed_attend(cache, x[:, :, :heads], out=out, ws=ws, add_scores=True, stream=stream)
        p = g10.g10_cache_plan_evictions(cache, 500, 4, 100, stream=stream)
        g10.g10_packed_evict(cache, p.moves, p.counts, stream=stream)
        return (p,) + g10.g10_packed_read(cache, 500, stream=stream)

    step(cache, out, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p, k, v = step(cache, out, ws)
    for to, source in ((cache.k, c.kc), (cache.v, c.vc), (cache.scales, c.scales), (cache.scores, c.scores)):
        to.view(torch.int8).copy_(source.view(torch.int8))
    x.copy_(torch.randn(4, new, heads + 4, 128, generator=gen).to(torch.bfloat16))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(2):
        g.replay()
        eager = g10.g10_packed_attend(other, x[:, :, :heads], stream=side)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    r, bound = reference(c, x[:, :, :heads].cpu())[:2]
    assert ((eager.cpu().double() - r.out).abs() <= bound).all()
    # the same twice, call by call
    mine = torch.empty_like(out)
    for _ in range(2):
        q, k2, v2 = step(other, mine, None)
    torch.cuda.synchronize()
    assert same(mine, out) and same(k, k2) and same(v, v2) and torch.equal(p.counts, q.counts)
    assert all(same(a, b) for a, b in zip((cache.k, cache.v, cache.scales, cache.scores), (other.k, other.v, other.scales, other.scores)))


def test_calls_of_two_threads(g10):
    import threading
    c = P.make_packed([900, 33, 400], 2, 128, 16, torch.bfloat16, "e4m3", 31)
    wrong = []
    want = {n: reference(c, queries(c, n, 4, n))[:2] for n in (1, 3)}

    def work(new):
        with torch.cuda.device(0), torch.cuda.stream(torch.cuda.Stream()):
            cache, dq = P.upload(g10, c), queries(c, new, 4, new).to(DEV)
            outs = [g10.g10_packed_attend(cache, dq) for _ in range(30)]
            torch.cuda.current_stream().synchronize()
            r, bound = want[new]
            wrong.extend(1 for out in outs if not ((out.cpu().double() - r.out).abs() <= bound).all())
            wrong.extend(1 for _ in range(int(cache.status.item() != 0)))

    threads = [threading.Thread(target=work, args=(n,)) for n in (1, 3, 1, 3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_what_is_read_back_attends_like_an_ordinary_cache(g10):
    """Whole pages that were read back are a cache of their own."""
    page, n = 16, 320
    c = P.make_packed([320, 50], 2, 128, page, torch.bfloat16, "int8", 3)
    cache = P.upload(g10, c)
    k, v = g10.g10_packed_read(cache, n)
    table = torch.arange(2 * n // page, dtype=torch.int32, device=DEV).view(2, -1)
    plain = g10.CacheBuffers(k.view(-1, page, 2, 128), v.view(-1, page, 2, 128), table, cache.lengths)
    q = queries(c, 30, 4, 1)
    out = g10.g10_cache_attend(plain, q.to(DEV)).cpu().double()
    P.values(c)
    P.rounded(c)
    r = O.attend(c, q, 128 ** -0.5)
    assert ((out - r.out).abs() <= O.attend_bounds(c, r)[0]).all()


@both
def test_a_conversation_within_a_budget(g10, code):
    """Prompts, eviction, then token after token with an eviction every few; each call is compared with the definitions applied to the device's state before it."""
    budget, page, kv, group, dim, room = 48, 16, 2, 3, 64, 8
    prompts = [70, 12, 130]
    gen = torch.Generator().manual_seed(3)
    columns = -(-(max(prompts) + 40) // page)
    pages = columns * 3 + 2
    table = torch.randperm(pages, generator=gen)[:columns * 3].view(3, columns).int()
    lengths = torch.tensor(prompts, dtype=torch.int32, device=DEV)
    seen = lengths.clone()
    angle = torch.arange(400, dtype=torch.float64)[:, None] * torch.pow(10000.0, -torch.arange(dim // 2, dtype=torch.float64) / (dim // 2))[None]
    cos, sin = angle.cos().float().to(DEV), angle.sin().float().to(DEV)
    cells = (pages, kv, page)
    codes = [torch.full((pages, page, kv, dim), 127, dtype=torch.int8, device=DEV).view(P.CODES[code]) for _ in range(2)]
    cache = g10.PackedBuffers(*codes, torch.full(cells + (2,), math.nan, device=DEV), table.to(DEV), lengths, seen=seen, scores=torch.full(cells, math.nan, device=DEV),
                              positions=torch.full(cells, -1, dtype=torch.int32, device=DEV))

    def host():
        from types import SimpleNamespace
        c = SimpleNamespace(kc=cache.k.cpu(), vc=cache.v.cpu(), scales=cache.scales.cpu(), table=table, lengths=lengths.cpu(), seen=seen.cpu(), page_size=page,
                            kv_heads=kv, head_dim=dim, dtype=torch.bfloat16, code=code, scores=cache.scores.cpu(), positions=cache.positions.cpu())
        P.values(c)
        return c

    def turn(new, counts):
        rows = torch.randn(3, new, kv * (group + 2), dim, generator=gen).to(torch.bfloat16).to(DEV)
        q = g10.g10_packed_append(cache, rows[:, :, kv * group:kv * (group + 1)], rows[:, :, kv * (group + 1):], rows[:, :, :kv * group], cos=cos, sin=sin, counts=counts.to(DEV))
        last = int(min(new, 5))
        at = (counts[:, None] - torch.minimum(counts, torch.tensor(last))[:, None] + torch.arange(last)[None]).clamp(max=new - 1).long().to(DEV)
        looks = torch.minimum(counts, torch.tensor(last)).int()
        q = q.gather(1, at[:, :, None, None].expand(-1, -1, kv * group, dim)).contiguous()
        c = host()
        r, b_out, _, rel = reference(c, q.cpu(), counts=looks)
        out = g10.g10_packed_attend(cache, q, counts=looks.to(DEV), add_scores=True).cpu().double()
        assert ((out - r.out).abs() <= b_out).all()
        after = cache.scores.cpu()
        for (s, h), w in r.booked.items():
            pg, pl = O.places(c, s, len(w))
            was = c.scores[pg, h, pl].double()
            assert ((after[pg, h, pl].double() - was - w).abs() <= w * float(rel[s].max()) + 2.0 ** -23 * (was + w)).all()

    def evict():
        c = host()
        p = g10.g10_cache_plan_evictions(cache, budget, 2, 8)
        moves, planned = O.plan(c, budget, 2, 8)
        g10.g10_packed_evict(cache, p.moves, p.counts)
        P.evict(c, moves)
        assert p.new_lengths.tolist() == planned
        assert same(cache.k, c.kc) and same(cache.v, c.vc) and same(cache.scales, c.scales) and same(cache.scores, c.scores)
        lengths.copy_(p.new_lengths)

    turn(max(prompts), torch.tensor(prompts, dtype=torch.int32))
    evict()
    for i in range(2 * room):
        lengths.add_(1)
        seen.add_(1)
        turn(1, torch.ones(3, dtype=torch.int32))
        if i % room == room - 1:
            evict()
    assert lengths.tolist() == [budget, 28, budget] and int(cache.status.item()) == 0


# ---- edges -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("new,group", [(1, 2), (1, 12), (4, 6)])
@pytest.mark.parametrize("pages", [0, 3])
@pytest.mark.parametrize("columns", [0, 2])
def test_nothing_to_look_at(g10, new, group, pages, columns):
    """Before the first page is given out.  Lengths of zero; or, where there are columns, lengths whose pages are none: read as zeros."""
    on = dict(device=DEV)
    k = torch.randint(-127, 128, (pages, 16, 2, 64), dtype=torch.int8, **on)
    cells = (pages, 2, 16)
    scores, positions, scales = torch.rand(cells, **on), torch.zeros(cells, dtype=torch.int32, **on), torch.rand(cells + (2,), **on)
    before = [x.clone() for x in (k, scores, scales)]
    table = torch.full((3, columns), -1, dtype=torch.int32, **on)
    for lengths in ([0, 0, 0],) if columns == 0 else ([0, 0, 0], [0, 5, 32]):
        cache = g10.PackedBuffers(k, k.clone(), scales, table, torch.tensor(lengths, dtype=torch.int32, **on), scores=scores, positions=positions)
        q = torch.randn(3, new, 2 * group, 64, **on).to(torch.bfloat16)
        out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:3], 9.0, **on)
        g10.g10_packed_attend(cache, q, add_scores=True, out=out, lse=lse)
        rows = torch.randn(3, new, 2, 64, **on).to(torch.bfloat16)
        g10.g10_packed_append(cache, rows, rows, q)
        p = g10.g10_cache_plan_evictions(cache, 4, 1, 1)
        g10.g10_packed_evict(cache, p.moves, p.counts)
        back = g10.g10_packed_read(cache, 40)
        torch.cuda.synchronize()
        assert int(cache.status.item()) == (0x400 if any(lengths) else 0)
        assert not out.any() and not back[0].any() and not back[1].any()
        for s, n in enumerate(lengths):                  # (a key of zeros has the logit 0)
            have = [n - min(new, n) + t + 1 for t in range(min(new, n))] + [0] * (new - min(new, n))
            want = torch.tensor([math.log(m) if m else -math.inf for m in have])
            got = lse[s].cpu()
            assert torch.allclose(got, want[:, None].expand_as(got), rtol=1e-6, atol=1e-6)
        assert same(k, before[0]) and same(scores, before[1]) and same(scales, before[2])


@pytest.mark.parametrize("code,dim,new,group", [("int8", 128, 20, 8), ("e4m3", 64, 1, 20), ("int8", 256, 3, 9)])
def test_a_wait_that_runs_out(monkeypatch, code, dim, new, group):
    """The test build, in which the first block of the kernels for many rows keeps one of its arrivals to itself (test_gpu_cache_edges.py): the call returns with the
    timeout bit, nothing is written out of place, and the next call is right."""
    import time
    from paper_2310_09443_b200 import binding, build
    monkeypatch.setattr(binding, "LIB_PATH", build.build(hooks=True))
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.delenv("G10_TEST_CACHE_MUTE", raising=False)
    binding.load_library()
    c = P.make_packed([9000, 700, 2500 + new], 8, dim, 64, torch.bfloat16, code, dim + group)
    q = queries(c, new, group, 3)
    dq = q.to(DEV)
    r, bound = reference(c, q)[:2]
    around = torch.full((2 * dq.numel(),), 7.0, dtype=dq.dtype, device=DEV)
    out = around[dq.numel() // 2:][:dq.numel()].view(dq.shape)
    size = binding.g10_packed_workspace_bytes(P.upload(binding, c), new, 8 * group, add_scores=True)
    ws = torch.zeros(size + 1024, dtype=torch.uint8, device=DEV)
    for mute in (0, 1, 2, 3, 4, 5, 6, 0):
        monkeypatch.setenv("G10_TEST_CACHE_MUTE", str(mute))
        cache = P.upload(binding, c)
        t0 = time.perf_counter()
        binding.g10_packed_attend(cache, dq, out=out, ws=ws[:size], add_scores=True)
        torch.cuda.synchronize()
        took = time.perf_counter() - t0
        assert int(cache.status.item()) == (0 if mute == 0 else 0x80), mute
        assert took < 1.0, (mute, took)
        assert (around[:dq.numel() // 2] == 7).all() and (around[dq.numel() // 2 + dq.numel():] == 7).all() and not ws[size:].any()
        assert same(cache.k, c.kc) and same(cache.v, c.vc)
        if mute == 0:
            assert ((out.cpu().double() - r.out).abs() <= bound).all()
