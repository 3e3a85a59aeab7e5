"""The cache of 8-bit rows at the edges of what is allowed, against the definitions in 64 bits (packed_oracle.py)."""
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
