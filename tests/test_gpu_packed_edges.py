"""The cache of 8-bit rows at the edges of what is allowed, against the definitions in 64 bits (packed_oracle.py)."""
import math

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


def test_read_of_as_many_tokens_as_there_may_be(g10):
    """2^31 - 65 tokens of one head of 16 dims (64 GB): the last ones are rows of the cache, all before them zeros."""
    tokens, length = 2 ** 31 - 65, 1000
    if torch.cuda.mem_get_info()[0] < 72 << 30:
        pytest.skip("wants 64 GB on the device")
    c = P.make_packed([length], 1, 16, 16, torch.bfloat16, "int8", 1)
    cache = P.upload(g10, c)
    k = torch.empty(1, tokens, 1, 16, dtype=torch.bfloat16, device=DEV)
    k[0, -20000:] = 5.0
    g10.g10_packed_read(cache, tokens, starts=torch.tensor([length - tokens], dtype=torch.int32, device=DEV), k=k)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    step = 1 << 27
    assert all(int(torch.count_nonzero(k[0, i:min(i + step, tokens - length)])) == 0 for i in range(0, tokens - length, step))
    pg, pl = O.places(c, 0, length)
    # (a code times its scale, rounded to 32 bits and to the type)
    assert torch.equal(k[0, -length:].cpu(), c.k[pg, pl].float().to(c.dtype))
    del k
    torch.cuda.empty_cache()


def test_evict_of_as_many_moves_as_there_may_be(g10):
    """2^31 - 65 moves (17 GB), none of which is one: each is looked at, and nothing is moved."""
    budget = 2 ** 31 - 65
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("wants 17 GB on the device")
    c = P.make_packed([100], 1, 16, 16, torch.bfloat16, "int8", 2)
    cache = P.upload(g10, c)
    moves = torch.full((1, 1, budget, 2), -1, dtype=torch.int32, device=DEV)
    counts = torch.tensor([[budget]], dtype=torch.int32, device=DEV)
    before = [x.clone() for x in (cache.k, cache.v, cache.scales, cache.scores)]
    g10.g10_packed_evict(cache, moves, counts)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0x2000
    for x, y in zip((cache.k, cache.v, cache.scales, cache.scores), before):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    del moves
    torch.cuda.empty_cache()


def attended(g10, c, q, counts=None, window=0, sinks=0, book=False):
    """The call's results, on the host."""
    cache = P.upload(g10, c)
    out, lse = torch.full(q.shape, 99.0, dtype=q.dtype, device=DEV), torch.full(q.shape[:3], 99.0, device=DEV)
    g10.g10_packed_attend(cache, q.to(DEV), counts=None if counts is None else counts.to(DEV), window=window, sinks=sinks, add_scores=book, out=out, lse=lse)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    return out.cpu(), lse.cpu(), cache


def queries(c, new, group, seed):
    gen = torch.Generator().manual_seed(seed + 77)
    return (2.0 * torch.randn(len(c.lengths), new, c.kv_heads * group, c.head_dim, generator=gen)).to(c.dtype)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("lengths,kv,dim,new,group", [([70, 90, 200], 2, 64, 4, 2), ([500, 40], 2, 128, 3, 5), ([9000, 300, 12000], 4, 64, 2, 4), ([700] * 90, 4, 128, 4, 1),
                                                      ([400, 90], 2, 256, 4, 4), ([500, 90], 2, 64, 9, 4), ([9000, 90, 300], 2, 128, 20, 8)])
def test_padding_beside_a_key_that_is_no_number(g10, lengths, kv, dim, new, group, code):
    """Head 0 of every sequence holds a key that is no number in its second slot: tokens that count are none there, those of padding are zeros all the same."""
    c = P.make_packed(lengths, kv, dim, 16, torch.bfloat16, code, 3)
    for s in range(len(lengths)):
        pg, pl = O.places(c, s, 2)
        c.scales[pg[1], 0, pl[1], 0] = math.nan
    counts = torch.tensor([(0, 1, new - 1, new)[s % 4] for s in range(len(lengths))], dtype=torch.int32)
    q = queries(c, new, group, 1)
    out, lse, _ = attended(g10, c, q, counts)
    for s, n in enumerate(counts.tolist()):
        assert (out[s, n:] == 0).all() and (lse[s, n:] == -math.inf).all(), s
        assert torch.isnan(out[s, :n, :group]).all() and torch.isnan(lse[s, :n, :group]).all()
        assert torch.isfinite(out[s, :n, group:].float()).all() and torch.isfinite(lse[s, :n, group:]).all()


def check_rows(c, q, out, lse, window=0, sinks=0):
    """Row by row against the definition.  The bounds are packed_oracle.py's, but for what a row does not see, which must not matter: a weight times its value's scale is rounded
    to fp16, half a step relatively or 2^-25 where the largest of the row's own is at least 2^10."""
    seqs, new, heads, dim = q.shape
    group, scale, step = heads // c.kv_heads, dim ** -0.5, O.half_step(c.dtype)
    for s, length in enumerate(c.lengths.tolist()):
        pg, pl = O.places(c, s, length)
        slot = torch.arange(length)
        for h in range(heads):
            k, v, (ks, vs), vc = c.k[pg, pl, h // group], c.v[pg, pl, h // group], c.scales[pg, h // group, pl].double().unbind(-1), c.vc[pg, pl, h // group].double()
            for t in range(new):
                at = length - new + t
                sees = slot <= at
                if window:
                    sees &= (slot < sinks) | (slot > at - window)
                row = q[s, t, h].double()
                x = k[sees] @ row * scale
                e = torch.exp(x - x.max())
                w = e / e.sum()
                n = len(x)
                slip = (k[sees].abs() @ row.abs()).max() * scale
                if c.code == "int8":
                    slip = slip + 128 * ks[sees].max() * row.abs().sum() * scale
                d = (2 * dim + 8) * 2.0 ** -23 * slip
                logs = torch.log2(vs[sees].clamp(min=2.0 ** -126)).abs().max()
                rel = 2 * d + 2.0 ** -21 + (n + 8) * 2.0 ** -23 + 2.0 ** -22 * (logs + 1)
                want = w @ v[sees]
                bound = (2.0 ** -11 + rel + (n + 8) * 2.0 ** -23) * (w @ v[sees].abs()) * 1.01 + 2.0 ** -34 * (w * vs[sees]).max() * vc[sees].abs().sum(0)
                bound = bound + step * (want.abs() + bound) + (2.0 ** -25 if c.dtype == torch.float16 else 0.0)
                assert ((out[s, t, h].double() - want).abs() <= bound).all(), (s, t, h)
                assert abs(float(lse[s, t, h]) - float(x.max() + torch.log(e.sum()))) <= float(d + rel + 2.0 ** -22 * abs(float(lse[s, t, h]))), (s, t, h)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("kind,least,most", [("bf16", 0, 60), ("bf16", -60, 119), ("fp16", -20, 8)])
@pytest.mark.parametrize("new,group,dim", [(2, 4, 64), (4, 4, 128), (9, 4, 64), (9, 4, 128), (33, 1, 128), (20, 8, 64), (5, 4, 256)])
def test_scales_of_values_that_a_row_does_not_see(g10, new, group, dim, kind, least, most, code):
    """The last tokens' values are 2^(most - least) larger than all others: only the tokens that see them may tell."""
    c = P.make_packed([150, 64 + new, 500], 1, dim, 16, O.TYPES[kind], code, new, garbage=False)
    c.scales[..., 1] *= 2.0 ** least
    for s, n in enumerate(c.lengths.tolist()):
        pg, pl = O.places(c, s, n)
        c.scales[pg[-1], 0, pl[-1], 1] = 2.0 ** most
        c.scales[pg[-2], 0, pl[-2], 1] = 2.0 ** ((least + most) // 2)
    P.values(c)
    q = queries(c, new, group, 2)
    out, lse, _ = attended(g10, c, q)
    check_rows(c, q, out, lse)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (20, 3), (70, 0)])
@pytest.mark.parametrize("new,group,dim", [(3, 4, 64), (9, 4, 128), (18, 8, 64), (6, 4, 256)])
def test_scales_of_values_outside_the_window(g10, new, group, dim, window, sinks, code):
    """Every token sees its own window only; large values stand in front of it, behind the sinks, and at the end."""
    c = P.make_packed([200, 70 + new, 400], 1, dim, 16, torch.bfloat16, code, new, garbage=False)
    for s, n in enumerate(c.lengths.tolist()):
        pg, pl = O.places(c, s, n)
        for j in (5, n // 2, n - new - window - 1, n - new - window, n - 1):
            if j >= sinks:
                c.scales[pg[j], 0, pl[j], 1] = 2.0 ** 60
    P.values(c)
    q = queries(c, new, group, 4)
    out, lse, _ = attended(g10, c, q, window=window, sinks=sinks)
    check_rows(c, q, out, lse, window, sinks)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("new,group,dim", [(1, 4, 64), (2, 8, 128), (9, 4, 64), (12, 8, 128), (6, 4, 256)])
def test_large_values_that_hardly_weigh(g10, new, group, dim, code):
    """Values 2^40 larger than the others' in slots that every row sees and whose weights are some 2^-90: next to nothing of the result, and no reason to lose bits of it."""
    c = P.make_packed([130, 64 + new, 700], 1, dim, 16, torch.bfloat16, code, new, garbage=False)
    q = queries(c, 1, 1, 5)
    q = (q + 0.1 * queries(c, new, group, 6)).to(c.dtype)
    for s, n in enumerate(c.lengths.tolist()):
        pg, pl = O.places(c, s, n)
        base = q[s, 0, 0].float()
        for j in (3, n // 2, n - new - 1):
            c.kc[pg[j], pl[j], 0] = (-torch.sign(base) * P.LARGEST[code]).to(c.kc.dtype)
            c.scales[pg[j], 0, pl[j], 0] = 62.0 / (P.LARGEST[code] * float(base.abs().sum()) * dim ** -0.5)
            c.scales[pg[j], 0, pl[j], 1] = 2.0 ** 40
    P.values(c)
    out, lse, _ = attended(g10, c, q)
    check_rows(c, q, out, lse)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("power", [-120, -60, 60, 117, 120, 123])
@pytest.mark.parametrize("new,group,dim", [(1, 4, 128), (2, 8, 64), (1, 3, 256)])
def test_queries_of_any_size(g10, new, group, dim, power, code):
    """Queries up to nearly the largest number of bf16 and keys as small: the logits are ordinary ones."""
    c = P.make_packed([90, 400], 2, dim, 16, torch.bfloat16, code, new)
    c.scales[..., 0] *= 2.0 ** -min(power, 119)
    P.values(c)
    q = (queries(c, new, group, 7).double() * 2.0 ** power).to(c.dtype)
    out, lse, _ = attended(g10, c, q)
    check_rows(c, q, out, lse)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("power", [-120, -60, 60, 117, 120, 123])
@pytest.mark.parametrize("new,group,dim", [(1, 4, 128), (9, 4, 64), (6, 6, 128), (40, 4, 64), (5, 4, 256)])
def test_queries_of_any_size_booked(g10, new, group, dim, power, code):
    """The same for more rows, and with the weights booked."""
    c = P.make_packed([90, 400], 2, dim, 16, torch.bfloat16, code, new)
    c.scales[..., 0] *= 2.0 ** -min(power, 119)
    P.values(c)
    q = (queries(c, new, group, 7).double() * 2.0 ** power).to(c.dtype)
    out, lse, cache = attended(g10, c, q, book=True)
    check_rows(c, q, out, lse)
    r = O.attend(c, q, dim ** -0.5)
    rel = P.attend_bounds(c, r, q, dim ** -0.5)[2].max()
    scores = cache.scores.cpu()
    for s, n in enumerate(c.lengths.tolist()):
        pg, pl = O.places(c, s, n)
        for h in range(2):
            was, got = c.scores[pg, h, pl].double(), scores[pg, h, pl].double()
            # (each weight off by rel, their sum in 32 bits, and the addition to what was there)
            assert ((got - was - r.booked[s, h]).abs() <= (rel + (new * group + 4) * 2.0 ** -23) * r.booked[s, h] + 2.0 ** -23 * got).all(), (s, h)


def test_ordinary_calls_take_anything_with_the_fields_of_a_cache(g10):
    """A program's own object that passes a cache's fields on: append, attend, plan and evict as with the cache itself."""
    class Layer:
        def __init__(self, cache):
            self.cache = cache

        def __getattr__(self, name):
            if name == "plan_ref":                       # (what a CacheBuffers did not always have)
                raise AttributeError(name)
            return getattr(self.cache, name)

    gen = torch.Generator().manual_seed(3)
    x = torch.randn(3, 1, 8, 64, generator=gen).to(torch.bfloat16).to(DEV)
    results = []
    for wrap in (lambda c: c, Layer):
        c = O.make_cache([200, 70, 90], 2, 64, 16, torch.bfloat16, 4, positions=True)
        cache = wrap(O.upload(g10, c))
        q = g10.g10_cache_append(cache, x[:, :, 4:6], x[:, :, 6:], x[:, :, :4])
        out = g10.g10_cache_attend(cache, q, add_scores=True)
        shared = g10.g10_cache_attend_shared(cache, q, torch.zeros(1, dtype=torch.int32, device=DEV))
        plan = g10.g10_cache_plan_evictions(cache, 80, sinks=4, recent=8)
        g10.g10_cache_evict(cache, plan.moves, plan.counts)
        torch.cuda.synchronize()
        assert int(cache.status.item()) == 0
        results.append([t.cpu() for t in (q, out, shared, plan.counts, plan.new_lengths, cache.k, cache.v, cache.scores, cache.positions)])
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    with pytest.raises(g10.G10Error):
        g10.g10_packed_evict(cache, plan.moves, plan.counts)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_read_rounds_the_product_in_32_bits(g10, kind, code):
    """Scales for which code times scale lies next to a tie of the type: what is read back is the product in 32 bits, rounded, as the call says."""
    dtype, dim = O.TYPES[kind], 64
    codes = torch.arange(3, 3 + dim).to(torch.int8) if code == "int8" else torch.arange(56, 56 + dim, dtype=torch.uint8).view(torch.float8_e4m3fn)
    ties = 1.0 + (2 * torch.arange(48) + 1).double() * (torch.finfo(dtype).eps / 2)
    c = P.make_packed([48], 1, dim, 16, dtype, code, 1)
    pg, pl = O.places(c, 0, 48)
    for side, which in ((0, 7), (1, 26)):
        (c.kc, c.vc)[side].view(torch.int8)[pg, pl, 0] = codes.view(torch.int8)
        c.scales[pg, 0, pl, side] = (ties / codes[which].double()).float()
    P.values(c)
    got = g10.g10_packed_read(P.upload(g10, c), 48)
    for x, exact in zip(got, (c.k, c.v)):
        exact = exact[pg, pl, 0]
        want = exact.float().to(dtype)
        assert torch.equal(x[0, :, 0].cpu(), want)
        # (one rounding of the exact product, to the nearer of the neighbours: not the same everywhere, or the cases would show nothing)
        step = torch.exp2(torch.floor(torch.log2(exact))) * torch.finfo(dtype).eps
        assert ((exact / step).round() * step != want.double()).any()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("how", ["grow", "shrink", "any", "jump"])
@pytest.mark.parametrize("lengths,new,group,dim", [([2600, 70], 1, 4, 64), ([2600, 70], 9, 4, 128), ([2600, 70], 5, 8, 64), ([900, 70], 33, 4, 64), ([1500, 70], 5, 4, 256), ([40000], 6, 4, 64)])
def test_scales_of_values_along_a_sequence(g10, lengths, new, group, dim, how, code):
    """Every tile's values are larger, or smaller, than those before, or any; logits grow towards the end for some rows and fall for others."""
    c = P.make_packed(lengths, 1, dim, 16, torch.bfloat16, code, new, garbage=False)
    q = queries(c, new, group, 8)
    gen = torch.Generator().manual_seed(9)
    for s, n in enumerate(lengths):
        pg, pl = O.places(c, s, n)
        at = torch.arange(n).double() / n
        power = {"grow": 160 * at - 80, "shrink": 80 - 160 * at, "any": torch.rand(n, generator=gen).double() * 160 - 80, "jump": torch.where(at < 0.5, -70.0, 70.0) * torch.where(at < 0.7, 1, -1)}[how]
        c.scales[pg, 0, pl, 1] = torch.exp2(power).float()
        keys = q[s, 0, 0].double()[None] * (at[:, None] * 2 - 1) + 0.2 * torch.randn(n, dim, generator=gen).double()
        kc, scale = P.packed(keys, code)
        c.kc.view(torch.int8)[pg, pl, 0] = kc.view(torch.int8)
        c.scales[pg, 0, pl, 0] = scale
    P.values(c)
    out, lse, _ = attended(g10, c, q)
    check_rows(c, q, out, lse)
