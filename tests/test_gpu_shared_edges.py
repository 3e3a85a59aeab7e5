"""Attention behind a shared beginning at the edges: scales of any sign, logits that are infinite, numbers that are none, for few rows a head, for some and for more than 128."""
import math
from types import SimpleNamespace

import pytest
import torch

import cache_oracle as O
from test_gpu_cache import queries
from test_gpu_shared import check, g10, make_shared  # noqa: F401  (g10: the fixture)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# sequences, new tokens, heads of a group, dims: 8, 36 and 300 rows a head, and more than 128 of heads that are too wide for the 256-row kernel
SIZES = [(2, 1, 4, 64), (3, 3, 4, 128), (5, 15, 4, 64), (5, 15, 4, 128), (75, 1, 4, 96), (3, 15, 4, 256)]


@pytest.mark.parametrize("scale", [-0.3, 0.0, -1e-3, 1.7])
@pytest.mark.parametrize("seqs,new,group,dim", SIZES)
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_scales(g10, kind, seqs, new, group, dim, scale):  # noqa: F811
    c = make_shared(640, [new + 13 * i for i in range(seqs)], 2, dim, 16, O.TYPES[kind], 5)
    check(g10, c, queries(c, new, group, 1), 640, scale=scale)


def attended(g10, c, q, common, counts):  # noqa: F811
    cache = O.upload(g10, c)
    out, lse = torch.full(q.shape, 99.0, dtype=q.dtype, device=DEV), torch.full(q.shape[:3], 99.0, device=DEV)
    g10.g10_cache_attend_shared(cache, q.to(DEV), torch.tensor([common], dtype=torch.int32, device=DEV), counts=counts.to(DEV), out=out, lse=lse)
    torch.cuda.synchronize()
    assert int(cache.status.item()) == 0
    return out.cpu().double(), lse.cpu().double()


def reference(c, q, counts):
    """cache_oracle.attend for keys that may be infinite (the size of a logit's error is that of the finite ones); rows that see nothing are zeros."""
    seqs, new, heads, dim = q.shape
    group, scale = heads // c.kv_heads, dim ** -0.5
    r = SimpleNamespace(out=torch.zeros(q.shape, dtype=torch.float64), lse=torch.full(q.shape[:3], -math.inf, dtype=torch.float64))
    r.weighed, r.all_v, r.slip, r.n_seen = torch.zeros_like(r.out), torch.zeros_like(r.out), torch.zeros(q.shape[:3], dtype=torch.float64), torch.zeros(q.shape[:3], dtype=torch.float64)
    for s, (length, count) in enumerate(zip(c.lengths.tolist(), counts.tolist())):
        pg, pl = O.places(c, s, length)
        for h in range(heads):
            k, v = c.k[pg, pl, h // group].double(), c.v[pg, pl, h // group].double()
            finite = torch.isfinite(k).all(-1)
            for t in range(count):
                n = length - count + t + 1
                row = q[s, t, h].double()
                x = k[:n] @ row * scale
                top = x.max()
                if top == -math.inf:
                    continue
                e = torch.exp(x - top)
                w = e / e.sum()
                i = (s, t, h)
                r.out[i], r.lse[i], r.weighed[i] = w @ v[:n], top + torch.log(e.sum()), w @ v[:n].abs()
                r.all_v[i], r.n_seen[i] = v[:n].abs().sum(0) / e.sum(), n
                r.slip[i] = (k[:n][finite[:n]].abs() @ row.abs()).max() * scale
    return r


def some_counts(seqs, new):
    return torch.tensor([(new, max(1, new - 1), 0)[i % 3] for i in range(seqs)], dtype=torch.int32)


@pytest.mark.parametrize("seqs,new,group,dim", SIZES)
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("where", ["first tiles", "last tiles", "all but a slot", "the beginning", "behind it"])
def test_logits_that_are_minus_infinity(g10, kind, where, seqs, new, group, dim):  # noqa: F811
    c = make_shared(640, [new + 13 * i for i in range(seqs)], 2, dim, 16, O.TYPES[kind], 6)
    q = (queries(c, new, group, 2).abs() + 0.25).to(c.dtype)
    part = {"first tiles": range(0, 400), "last tiles": range(250, 640), "all but a slot": [j for j in range(640) if j != 333], "the beginning": range(640)}.get(where)
    for s in range(seqs):
        n = int(c.lengths[s])
        pg, pl = O.places(c, s, n)
        at = torch.tensor(list(range(640, n) if part is None else part))
        c.k[pg[at], pl[at]] = -math.inf
    counts = some_counts(seqs, new)
    out, lse = attended(g10, c, q, 640, counts)
    r = reference(c, q, counts)
    b_out, b_lse, _ = O.attend_bounds(c, r)
    nothing = torch.isinf(r.lse)
    assert (out[nothing] == 0).all() and torch.equal(torch.isinf(lse), nothing)
    assert ((out - r.out).abs() <= b_out).all() and ((lse - r.lse).abs() <= b_lse)[~nothing].all()


@pytest.mark.parametrize("seqs,new,group,dim", SIZES)
def test_logits_that_are_all_minus_infinity(g10, seqs, new, group, dim):  # noqa: F811
    c = make_shared(640, [new + 13 * i for i in range(seqs)], 2, dim, 16, torch.bfloat16, 7)
    c.k[:, :, 0] = -math.inf
    counts = some_counts(seqs, new)
    q = (queries(c, new, group, 3).abs() + 0.25).to(c.dtype)
    out, lse = attended(g10, c, q, 640, counts)
    assert (out[:, :, :group] == 0).all() and (lse[:, :, :group] == -math.inf).all()
    real = torch.arange(new)[None] < counts[:, None]
    assert torch.isfinite(out).all() and torch.equal(torch.isfinite(lse[:, :, group]), real)


@pytest.mark.parametrize("seqs,new,group,dim", SIZES)
@pytest.mark.parametrize("slot", [0, 70, 639])
@pytest.mark.parametrize("what", ["key", "infinite key", "value"])
def test_a_row_of_the_beginning_that_is_no_number(g10, what, slot, seqs, new, group, dim):  # noqa: F811
    """... or an infinite logit: none for every token's rows of that head (of a value: that dimension), all others as ever, padding zeros."""
    c = make_shared(640, [new + 13 * i for i in range(seqs)], 2, dim, 16, torch.bfloat16, 8)
    q = (queries(c, new, group, 4).abs() + 0.25).to(c.dtype)
    counts = some_counts(seqs, new)
    pg, pl = O.places(c, 0, 640)
    r = reference(c, q, counts)
    if what == "value":
        c.v[pg[slot], pl[slot], 0, 5] = math.nan
    else:
        c.k[pg[slot], pl[slot], 0] = math.nan if what == "key" else math.inf
    out, lse = attended(g10, c, q, 640, counts)
    bad = torch.zeros(out.shape, dtype=torch.bool)
    real = torch.arange(new)[None] < counts[:, None]
    bad[:, :, :group, 5 if what == "value" else slice(None)] = real[:, :, None] if what == "value" else real[:, :, None, None]
    assert torch.equal(torch.isnan(out), bad)
    b_out, b_lse, _ = O.attend_bounds(c, r)
    assert ((out - r.out).abs() <= b_out)[~bad].all() and (out[~real] == 0).all() and (lse[~real] == -math.inf).all()
    fine = real[:, :, None].expand(lse.shape).clone()
    if what != "value":
        assert torch.isnan(lse[:, :, :group][real]).all()
        fine[:, :, :group] = False
    assert ((lse - r.lse).abs() <= b_lse)[fine].all()
