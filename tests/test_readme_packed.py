"""The README's blocks on the cache of 8-bit rows and on a shared beginning run."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def block(name):
    with open(os.path.join(ROOT, "README.md")) as f:
        found = [x for x in re.findall(r"```python\n(.*?)```", f.read(), re.S) if name in x]
    assert len(found) == 1
    return found[0]


@pytest.mark.gpu
def test_they_run():
    import torch
    from paper_2310_09443_b200 import binding as g10, build
    build.build()
    page, heads, kv_heads, dim, seqs, budget = 16, 32, 8, 128, 8, 128
    columns = 14
    pages = seqs * columns
    names = dict(torch=torch, g10=g10, page=page, kv_heads=kv_heads, dim=dim, pages=pages, budget=budget, cells=(pages, kv_heads, page),
                 page_table=torch.arange(pages, dtype=torch.int32, device="cuda").view(seqs, -1), lengths=torch.full((seqs,), 100, dtype=torch.int32, device="cuda"),
                 seen=torch.full((seqs,), 100, dtype=torch.int32, device="cuda"), qw=torch.ones(dim, dtype=torch.bfloat16, device="cuda"),
                 kw=torch.ones(dim, dtype=torch.bfloat16, device="cuda"), cos=torch.ones(300, dim // 2, device="cuda"), sin=torch.zeros(300, dim // 2, device="cuda"))
    # (a prompt is appended whole, and looked at from its tokens)
    for name, n in (("new_q", heads), ("new_k", kv_heads), ("new_v", kv_heads)):
        names[name] = torch.randn(seqs, 100, n, dim, device="cuda").to(torch.bfloat16)
    exec(block("g10_packed_append"), names)
    torch.cuda.synchronize()
    assert int(names["packed"].status.item()) == 0 and torch.isfinite(names["out"]).all()
    assert names["plan"].counts.sum().item() == 0 and names["last_k"].shape == (seqs, 64, kv_heads, dim)
    # what was read back is what was appended, to half a step of a row's largest element
    error = (names["last_v"].float() - names["new_v"][:, 36:].float()).abs().amax(-1)
    assert (error <= names["new_v"][:, 36:].float().abs().amax(-1) * (0.5 / 127 + 2.0 ** -8)).all()
    k, v = (torch.randn(pages, page, kv_heads, dim, device="cuda").to(torch.bfloat16) for _ in range(2))
    names["page_table"][:, :4] = names["page_table"][:1, :4]
    names.update(beginning=70, cache=g10.CacheBuffers(k, v, names["page_table"], names["lengths"]), q=names["new_q"][:, :1].contiguous())
    exec(block("g10_cache_attend_shared"), names)
    plain = g10.g10_cache_attend(names["cache"], names["q"])
    assert int(names["shared"].item()) == 64 and (names["out"].float() - plain.float()).abs().max() < 0.02
