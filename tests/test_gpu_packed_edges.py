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
