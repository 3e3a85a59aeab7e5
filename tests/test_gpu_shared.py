"""Attention of a batch behind a shared beginning against the definitions in 64 bits (cache_oracle.py)."""
import math

import pytest
import torch

import cache_oracle as O
from test_gpu_cache import queries, same

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def g10():
    from paper_2310_09443_b200 import binding, build
    build.build()
    binding.load_library()
    return binding


def make_shared(common, own, kv, dim, page, dtype, seed, **more):
    """A cache whose sequences share `common` slots (whole pages) and have `own` slots each behind them."""
    assert common % page == 0
    c = O.make_cache([common + n for n in own], kv, dim, page, dtype, seed, **more)
    c.table[1:, :common // page] = c.table[0, :common // page]
    return c


def check(g10, c, q, common, counts=None, strided=False, scale=None, said=None, status=0):
    cache = O.upload(g10, c)
    dq = q.to(DEV)
    if strided:
        wide = torch.full(q.shape[:2] + (q.shape[2] + 3, q.shape[3]), math.nan, dtype=q.dtype, device=DEV)
        wide[:, :, 1:-2] = dq
        dq = wide[:, :, 1:-2]
    scale = c.head_dim ** -0.5 if scale is None else scale
    out, lse = torch.full(q.shape, 99.0, dtype=q.dtype, device=DEV), torch.full(q.shape[:3], 99.0, device=DEV)
    shared = torch.tensor([common if said is None else said], dtype=torch.int32, device=DEV)
    g10.g10_cache_attend_shared(cache, dq, shared, scale=scale, counts=None if counts is None else counts.to(DEV), out=out, lse=lse)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == status
    r = O.attend(c, q, scale, counts=counts)
    b_out, b_lse, _ = O.attend_bounds(c, r)
    out, lse = out.cpu().double(), lse.cpu().double()
    nothing = torch.isinf(r.lse)
    assert (out[nothing] == 0).all() and torch.equal(torch.isinf(lse), nothing)
    assert ((out - r.out).abs() <= b_out).all() and ((lse - r.lse).abs() <= b_lse)[~nothing].all()


@pytest.mark.parametrize("dim", [8, 64, 72, 80, 96, 128, 136, 192, 256])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("new,group", [(1, 2), (1, 5), (3, 7), (9, 5)])
def test_head_dims(g10, dim, kind, new, group):
    c = make_shared(208, [new, new + 1, 70 + new, 200], 2, dim, 16, O.TYPES[kind], dim)
    check(g10, c, queries(c, new, group, dim), 208)


@pytest.mark.parametrize("common", [0, 16, 48, 64, 112, 128, 192, 640, 4096])
@pytest.mark.parametrize("seqs,new,group", [(1, 1, 1), (3, 1, 4), (20, 1, 8), (5, 20, 3), (70, 2, 2), (129, 1, 1), (32, 1, 8), (33, 1, 8), (100, 1, 4)])
def test_lengths_of_the_beginning(g10, common, seqs, new, group):
    own = [new + (37 * i) % 90 for i in range(seqs)]
    c = make_shared(common, own, 2, 64, 16, torch.bfloat16, common + seqs)
    check(g10, c, queries(c, new, group, seqs), common)
    if common >= 64:                                     # less than is shared may be said, as far as a page's middle
        check(g10, c, queries(c, new, group, seqs), common, said=common - 39)


@pytest.mark.parametrize("page,common", [(1, 201), (7, 175), (24, 192), (100, 300), (256, 256)])
@pytest.mark.parametrize("layout", ["slots", "heads", "wide"])
def test_pages_and_strides(g10, page, common, layout):
    c = make_shared(common, [1, 5, 97, 100, 333], 2, 128, page, torch.float16, page, layout=layout)
    check(g10, c, queries(c, 1, 4, page), common, strided=True)
    check(g10, c, queries(c, 5, 4, page), common, counts=torch.tensor([1, 5, 0, 3, 5], dtype=torch.int32), strided=True)


@pytest.mark.parametrize("new,group", [(1, 4), (4, 4), (16, 2), (30, 6)])
def test_padding_and_sequences_without_tokens(g10, new, group):
    """Sequences without new tokens may be of any length, shorter than the beginning too; padding may hold anything."""
    c = make_shared(320, [new, new + 3, 100 + new, new], 2, 64, 16, torch.bfloat16, new)
    counts = torch.tensor([0, max(1, new // 2), new, 0], dtype=torch.int32)
    c.lengths[3] = 10
    q = queries(c, new, group, 1)
    for s, n in enumerate(counts.tolist()):
        q[s, n:] = math.nan
    check(g10, c, q, 320, counts=counts)
    check(g10, c, q, 320, counts=torch.zeros(4, dtype=torch.int32))


def test_more_than_is_shared_is_reported(g10):
    """... and as much is taken as can be."""
    c = make_shared(320, [40, 9, 100], 2, 64, 16, torch.bfloat16, 2)
    q = queries(c, 2, 4, 1)
    # (sequence 1 holds 327 slots before its new tokens: 320 are whole tiles)
    for said in (328, 400, 2 ** 31 - 1):
        check(g10, c, q, 320, said=said, status=0x800)
    for said in (-1, -2 ** 31):
        check(g10, c, q, 320, said=said, status=0x800)


@pytest.mark.parametrize("new", [1, 6, 40])
def test_values_that_are_not_finite_are_seen_by_their_rows_alone(g10, new):
    c = make_shared(128, [new + 30, new + 70], 2, 64, 16, torch.float16, 6)
    q = queries(c, new, 4, 2)
    pg, pl = O.places(c, 1, int(c.lengths[1]))
    for x in (c.k, c.v):
        x[pg[-1], pl[-1]] = math.nan                     # the last token of sequence 1
    cache = O.upload(g10, c)
    lse = torch.empty(q.shape[:3], device=DEV)
    out = g10.g10_cache_attend_shared(cache, q.to(DEV), torch.tensor([128], dtype=torch.int32, device=DEV), lse=lse).cpu()
    bad = torch.zeros(q.shape[:2], dtype=torch.bool)
    bad[1, new - 1] = True
    assert torch.equal(torch.isnan(out).any(-1).any(-1), bad)
    c.k[torch.isnan(c.k)] = 0
    c.v[torch.isnan(c.v)] = 0
    r = O.attend(c, q, 0.125)
    assert ((out.double() - r.out).abs() <= O.attend_bounds(c, r)[0])[~bad].all()


def test_infinite_logits(g10):
    """A beginning that weighs nothing, or all."""
    c = make_shared(128, [40, 70], 2, 64, 16, torch.float16, 6)
    q = queries(c, 1, 4, 2).abs()
    for sign in (1.0, -1.0):
        for part in (0, 1):
            d = make_shared(128, [40, 70], 2, 64, 16, torch.float16, 6)
            for s in range(2):
                pg, pl = O.places(d, s, int(d.lengths[s]))
                where = slice(0, 128) if part == 0 else slice(128, None)
                d.k[pg[where], pl[where]] = sign * 200.0
            check(g10, d, q, 128)


@pytest.mark.parametrize("seqs,new,group,kv,dim,common", [(64, 1, 8, 2, 128, 9000), (33, 3, 5, 1, 96, 5000), (2, 1, 1, 8, 64, 20000), (9, 60, 8, 1, 128, 3000), (3, 2, 6, 1, 256, 2500),
                                                           (40, 1, 4, 3, 64, 7000), (130, 1, 4, 2, 128, 1280), (65, 2, 2, 2, 40, 6500), (300, 1, 1, 2, 112, 10000)])
def test_long(g10, seqs, new, group, kv, dim, common):
    page = 20
    c = make_shared(common // page * page, [new + (131 * i) % 400 for i in range(seqs)], kv, dim, page, torch.bfloat16, seqs)
    check(g10, c, queries(c, new, group, 3), common // page * page)


def test_later_beginnings_outweigh_all_before(g10):
    c = make_shared(1280, [30] * 12, 1, 64, 16, torch.float16, 2, garbage=False)
    q = queries(c, 1, 8, 4)
    q[:] = q[:1, :, :1]
    pg, pl = O.places(c, 0, 1280)
    c.k[pg, pl, 0] = (q[0, 0, 0].double()[None] * torch.linspace(0.0, 3.0, 1280, dtype=torch.float64)[:, None]).half()
    check(g10, c, q, 1280)


def test_the_workspace_may_hold_anything_and_results_repeat(g10):
    c = make_shared(2048, [300, 40, 90] * 5, 2, 128, 16, torch.bfloat16, 3)
    cache, dq = O.upload(g10, c), queries(c, 2, 4, 1).to(DEV)
    shared = torch.tensor([2048], dtype=torch.int32, device=DEV)
    n = g10.g10_cache_shared_workspace_bytes(cache, 2, 8)
    first = None
    for fill in (0, 255, 127):
        ws = torch.full((n,), fill, dtype=torch.uint8, device=DEV)
        out = g10.g10_cache_attend_shared(cache, dq, shared, ws=ws)
        assert first is None or same(out, first)
        first = out


@pytest.mark.parametrize("new,group", [(1, 4), (5, 6)])
def test_captured_beside_others(g10, new, group):
    """Two captured calls with a workspace each, replayed side by side after the lengths and the beginning have moved on, beside eager calls on a third stream."""
    c = make_shared(640, [300, 40, 90, 500] * 3, 2, 128, 16, torch.bfloat16, 3)
    cache = O.upload(g10, c)
    q = queries(c, new, group, 1)
    dq = q.to(DEV)
    shared = torch.tensor([640], dtype=torch.int32, device=DEV)
    graphs = []
    for i in range(2):
        out = torch.empty_like(dq)
        ws = torch.empty(g10.g10_cache_shared_workspace_bytes(cache, new, 2 * group), dtype=torch.uint8, device=DEV)
        g10.g10_cache_attend_shared(cache, dq, shared, out=out, ws=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            g10.g10_cache_attend_shared(cache, dq, shared, out=out, ws=ws)
        graphs.append((g, out, torch.cuda.Stream(), ws))     # (a graph does not keep its workspace: a capture gives cached memory back)
    side = torch.cuda.Stream()
    full = c.lengths.clone()
    for cut, common in ((0, 640), (20, 320), (5, 0)):
        c.lengths = full - cut
        cache.lengths.copy_(c.lengths)
        shared.fill_(common)
        torch.cuda.synchronize()
        for _ in range(10):
            for g, _, stream, _ in graphs:
                with torch.cuda.stream(stream):
                    g.replay()
            eager = g10.g10_cache_attend_shared(cache, dq, shared, stream=side)
        torch.cuda.synchronize()
        r = O.attend(c, q, 128 ** -0.5)
        bound = O.attend_bounds(c, r)[0]
        for out in [eager] + [x[1] for x in graphs]:
            assert ((out.cpu().double() - r.out).abs() <= bound).all()
    assert int(cache.status.item()) == 0


def test_many_sequences(g10):
    """More sequences than the checking block has threads; a run of append and attend."""
    seqs, page = 1500, 16
    c = make_shared(256, [1 + i % 50 for i in range(seqs)], 1, 64, page, torch.bfloat16, 4)
    cache = O.upload(g10, c)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(seqs, 1, 4, 64, generator=gen).to(torch.bfloat16).to(DEV)
    q = g10.g10_cache_append(cache, x[:, :, 2:3], x[:, :, 3:], x[:, :, :2])
    out = g10.g10_cache_attend_shared(cache, q, torch.tensor([256], dtype=torch.int32, device=DEV))
    plain = g10.g10_cache_attend(cache, q)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    c.k, c.v = cache.k.cpu(), cache.v.cpu()
    r = O.attend(c, q.cpu(), 0.125)
    bound = O.attend_bounds(c, r)[0]
    for o in (out, plain):
        assert ((o.cpu().double() - r.out).abs() <= bound).all()


@pytest.mark.parametrize("new", [1, 3, 20])
def test_offsets_beyond_32_bits(g10, new):
    """Rows more than 2^32 bytes into the pool, for 12, 36 and 240 rows a head, called on a stream of its own."""
    page, kv, dim = 64, 8, 128
    pages = (1 << 32) // (page * kv * dim * 2) + 60
    c = make_shared(320, [new, 33, 90], kv, dim, page, torch.bfloat16, 8)
    pool = [torch.empty(pages, page, kv, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    shift = pages - c.k.shape[0]
    for to, x in zip(pool, (c.k, c.v)):
        to[shift:] = x.to(DEV)
    table = torch.where(c.table >= 0, c.table + shift, c.table)
    cache = g10.CacheBuffers(*pool, table.to(DEV), c.lengths.to(DEV))
    q = queries(c, new, 4, new)
    dq, shared = q.to(DEV), torch.tensor([320], dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    out = g10.g10_cache_attend_shared(cache, dq, shared, stream=stream)
    stream.synchronize()
    assert int(cache.status.item()) == 0
    r = O.attend(c, q, dim ** -0.5)
    assert ((out.cpu().double() - r.out).abs() <= O.attend_bounds(c, r)[0]).all()


def test_bad_pages_of_the_beginning(g10):
    c = make_shared(128, [20, 40], 2, 64, 16, torch.bfloat16, 6)
    q = queries(c, 1, 4, 1).to(DEV)
    shared = torch.tensor([128], dtype=torch.int32, device=DEV)
    for page in (-1, -2 ** 31, c.k.shape[0], 2 ** 31 - 1):
        c.table[0, 2] = page
        cache = O.upload(g10, c)
        g10.g10_cache_attend_shared(cache, q, shared)
        assert int(cache.status.item()) == 0x400
    c.table[0, 2] = c.table[0, 1]
    for length in (-1, -2 ** 31, 10 ** 6):
        c.lengths[1] = length
        cache = O.upload(g10, c)
        g10.g10_cache_attend_shared(cache, q, shared)
        assert int(cache.status.item()) == 0x800


def test_refusals(g10):
    c = make_shared(128, [20, 40], 2, 64, 16, torch.bfloat16, 6)
    cache = O.upload(g10, c)
    q = queries(c, 1, 4, 1).to(DEV)
    shared = torch.tensor([128], dtype=torch.int32, device=DEV)
    for x, sh, kw in [(q.float(), shared, {}), (q[:1], shared, {}), (q[:, :, :7], shared, {}), (q, shared.cpu(), {}), (q, shared.long(), {}), (q, shared.expand(2), {}),
                      (q, shared, dict(ws=torch.empty(64, dtype=torch.uint8, device=DEV))), (q, shared, dict(out=q.float())), (q, shared, dict(lse=shared)),
                      (q, shared, dict(counts=shared)), (q, shared, dict(scale=math.inf)), (torch.zeros(2, 300, 8, 64, dtype=q.dtype, device=DEV), shared, {})]:
        with pytest.raises(g10.G10Error):
            g10.g10_cache_attend_shared(cache, x, sh, **kw)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0


@pytest.mark.parametrize("dim,seqs,new,group", [(128, 40, 1, 8), (64, 40, 1, 8), (192, 20, 2, 4), (128, 6, 3, 6)])
def test_a_wait_that_runs_out(monkeypatch, dim, seqs, new, group):
    """The test build, in which the first block of the kernels for many rows keeps one of its arrivals to itself (test_gpu_cache_edges.py): the call returns with the
    timeout bit, nothing is written out of place, and the next call is right."""
    import time
    from paper_2310_09443_b200 import binding, build
    monkeypatch.setattr(binding, "LIB_PATH", build.build(hooks=True))
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.delenv("G10_TEST_CACHE_MUTE", raising=False)
    binding.load_library()
    common = 25600                                       # (a block has more than one tile: the second is the one that is kept)
    c = make_shared(common, [new + (29 * i) % 200 for i in range(seqs)], 2, dim, 64, torch.bfloat16, dim)
    q = queries(c, new, group, 3)
    dq = q.to(DEV)
    r = O.attend(c, q, dim ** -0.5)
    bound = O.attend_bounds(c, r)[0]
    shared = torch.tensor([common], dtype=torch.int32, device=DEV)
    around = torch.full((2 * dq.numel(),), 7.0, dtype=dq.dtype, device=DEV)
    out = around[dq.numel() // 2:][:dq.numel()].view(dq.shape)
    size = binding.g10_cache_shared_workspace_bytes(O.upload(binding, c), new, 2 * group)
    ws = torch.zeros(size + 1024, dtype=torch.uint8, device=DEV)
    for mute in (0, 1, 2, 3, 6, 0):
        monkeypatch.setenv("G10_TEST_CACHE_MUTE", str(mute))
        cache = O.upload(binding, c)
        t0 = time.perf_counter()
        binding.g10_cache_attend_shared(cache, dq, shared, out=out, ws=ws[:size])
        torch.cuda.synchronize()
        took = time.perf_counter() - t0
        assert int(cache.status.item()) == (0 if mute == 0 else 0x80), mute
        assert took < 1.0, (mute, took)
        assert (around[:dq.numel() // 2] == 7).all() and (around[dq.numel() // 2 + dq.numel():] == 7).all() and not ws[size:].any()
        assert same(cache.k, c.k) and same(cache.v, c.v)
        if mute == 0:
            assert ((out.cpu().double() - r.out).abs() <= bound).all()
