"""The README's quick start of the key-value cache: its pool has room for what it does, and it runs."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def block():
    with open(os.path.join(ROOT, "README.md")) as f:
        found = [x for x in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "g10_cache_append" in x]
    assert len(found) == 1
    return found[0]


def test_the_pool_has_room_beyond_the_budget():
    """A sequence at its budget takes at least one more token before it can be evicted."""
    numbers = {}
    for line in block().splitlines():
        if "torch" in line:
            break
        exec(line, numbers)
    assert numbers["pages"] >= numbers["seqs"] * -(-(numbers["budget"] + 1) // numbers["page"])


@pytest.mark.gpu
def test_it_runs():
    import torch
    from paper_2310_09443_b200 import binding as g10, build
    build.build()
    names = dict(torch=torch, g10=g10)
    exec(block(), names)
    seqs, heads, kv_heads, dim, budget, room = (names[x] for x in ("seqs", "heads", "kv_heads", "dim", "budget", "room"))
    gen = torch.Generator(device="cuda").manual_seed(1)
    angle = torch.rand(budget + 3 * room, dim // 2, generator=gen, device="cuda") * 6.28
    names.update(qw=torch.ones(dim, dtype=torch.bfloat16, device="cuda"), kw=torch.ones(dim, dtype=torch.bfloat16, device="cuda"), cos=angle.cos(), sin=angle.sin())
    for i in range(budget + 3 * room):
        for name, n in (("new_q", heads), ("new_k", kv_heads), ("new_v", kv_heads)):
            names[name] = torch.randn(seqs, 1, n, dim, generator=gen, device="cuda").to(torch.bfloat16)
        out = names["step"]()
        if int(i + 1) % room == 0:
            names["evict"]()
    assert torch.isfinite(out).all() and int(names["cache"].status.item()) == 0
    assert names["lengths"].tolist() == [budget] * seqs and names["seen"].tolist() == [budget + 3 * room] * seqs
    assert torch.isfinite(names["cache"].scores).all()
