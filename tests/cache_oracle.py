"""The calls on the key-value cache restated in 64 bits, sequence by sequence and head by head, and inputs for them.

Everything is computed from the definitions with torch in float64 on the host; nothing is shared with the library."""
import math
from types import SimpleNamespace

import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def half_step(dtype):
    """Largest relative error of one rounding to the type."""
    return torch.finfo(dtype).eps / 2


def make_cache(lengths, kv_heads, head_dim, page_size, dtype, seed, columns=None, spare=3, layout="slots", scores=True, positions=False, garbage=True):
    """A cache on the host: pages in random order, NaN wherever no token stands (and -1 in the table behind the sequences)."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator().manual_seed(seed)
    need = [-(-n // page_size) for n in lengths]
    columns = max(need + [1]) if columns is None else columns
    pages = sum(need) + spare
    order = rng.permutation(pages)
    table = np.full((len(lengths), columns), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    shape = (pages, page_size, kv_heads, head_dim)
    k, v = (torch.randn(shape, generator=gen).to(dtype) for _ in range(2))
    owned = torch.zeros(pages, page_size, dtype=torch.bool)
    for s, n in enumerate(lengths):
        for j in range(need[s]):
            owned[table[s, j], :min(page_size, n - j * page_size)] = True
    if garbage:
        k[~owned], v[~owned] = math.nan, math.nan
    c = SimpleNamespace(k=k, v=v, table=torch.from_numpy(table), lengths=torch.tensor(lengths, dtype=torch.int32), seen=None, page_size=page_size,
                        kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, layout=layout)
    cells = (pages, kv_heads, page_size)
    c.scores = torch.rand(cells, generator=gen) if scores else None
    c.positions = None
    if positions:
        c.positions = torch.full(cells, -7, dtype=torch.int32)
        for s, n in enumerate(lengths):
            for h in range(kv_heads):
                pg, pl = places(c, s, n)
                c.positions[pg, h, pl] = torch.arange(n, dtype=torch.int32)
    return c


def places(c, s, n):
    """Page and place of the first n slots of sequence s."""
    slot = torch.arange(n)
    return c.table[s].long()[slot // c.page_size], slot % c.page_size


def upload(g10, c, device="cuda:0", **more):
    """The cache on the device (in the layout that it asks for) as CacheBuffers."""
    def rows(x):
        if c.layout == "heads":                        # [pages, kv_heads, page_size, head_dim] seen as [pages, page_size, kv_heads, head_dim]
            return x.transpose(1, 2).contiguous().to(device).transpose(1, 2)
        if c.layout == "wide":                         # rows of a larger tensor
            big = torch.full((x.shape[0], 2, x.shape[1], x.shape[2], x.shape[3] + 8), math.nan, dtype=x.dtype, device=device)
            big[:, 1, :, :, 8:] = x.to(device)
            return big[:, 1, :, :, 8:]
        return x.to(device)
    on = lambda x: None if x is None else x.to(device)
    return g10.CacheBuffers(rows(c.k), rows(c.v), on(c.table), on(c.lengths), seen=on(c.seen), scores=on(c.scores), positions=on(c.positions), **more)


def counts_of(c, counts, new):
    have = c.lengths.tolist()
    want = [new] * len(have) if counts is None else counts.tolist()
    return [min(w, n) for w, n in zip(want, have)]


def attend(c, q, scale, window=0, sinks=0, counts=None):
    """out, lse, booked weights by (sequence, head) and, for the bounds: sum w |v|, sum |v| over what is seen and the error of a logit."""
    seqs, new, heads, dim = q.shape
    group = heads // c.kv_heads
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64)
    weighed, all_v = torch.zeros_like(out), torch.zeros_like(out)
    slip = torch.zeros(q.shape[:3], dtype=torch.float64)
    n_seen = torch.zeros(q.shape[:3], dtype=torch.float64)
    booked = {}
    for s, (length, count) in enumerate(zip(c.lengths.tolist(), counts_of(c, counts, new))):
        pg, pl = places(c, s, length)
        slot = torch.arange(length)
        for h in range(c.kv_heads):
            k, v = c.k[pg, pl, h].double(), c.v[pg, pl, h].double()
            total = torch.zeros(length, dtype=torch.float64)
            for t in range(count):
                p = length - count + t
                sees = slot <= p
                if window:
                    sees &= (slot < sinks) | (slot > p - window)
                ks, vs = k[sees], v[sees]
                for g in range(group):
                    row = q[s, t, h * group + g].double()
                    x = ks @ row * scale
                    top = x.max()
                    e = torch.exp(x - top)
                    w = e / e.sum()
                    i = (s, t, h * group + g)
                    out[i] = w @ vs
                    lse[i] = top + torch.log(e.sum())
                    weighed[i], all_v[i] = w @ vs.abs(), vs.abs().sum(0) / e.sum()
                    slip[i] = (ks.abs() @ row.abs()).max() * abs(scale)      # (an error has no sign: the size of the scale)
                    n_seen[i] = len(x)
                    total[sees] += w
            booked[s, h] = total
    return SimpleNamespace(out=out, lse=lse, booked=booked, weighed=weighed, all_v=all_v, slip=slip, n_seen=n_seen)


def attend_bounds(c, r):
    """How far out, lse and a weight (relatively) may be off.

    A product of two stored values is exact in 32 bits; adding D of them costs at most D * 2^-23 of the sum of their sizes (units that add with
    truncation included), so a logit is off by d = (D + 4) * 2^-23 * scale * sum |q k| (scaling and the change to base 2 among the 4).  A weight is
    then off by the factor 1 + 2 d (its own logit, and the sum's), by 2^-21 for two exponentials, and by (n + 8) * 2^-23 for the sum of n of
    them.  `out` has each weight rounded to the type (half a step relative, or half the smallest subnormal of fp16 before the division), n
    sums in 32 bits, and its own rounding."""
    step = half_step(c.dtype)
    d = (c.head_dim + 4) * 2.0 ** -23 * r.slip
    rel = 2 * d + 2.0 ** -21 + (r.n_seen + 8) * 2.0 ** -23
    tiny = 2.0 ** -25 if c.dtype == torch.float16 else 0.0
    out = (step + rel[..., None] + (r.n_seen[..., None] + 8) * 2.0 ** -23) * r.weighed * 1.01 + tiny * r.all_v
    out = out + step * (r.out.abs() + out) + (2.0 ** -25 if c.dtype == torch.float16 else 0.0)
    lse = d + rel + 2.0 ** -22 * r.lse.abs()
    return out, lse, rel


def turned(x, weight, eps, cos, sin, position, interleaved):
    x = x.double()
    if weight is not None:
        x = x / math.sqrt(float((x * x).mean()) + eps) * weight.double()
    if cos is None:
        return x
    half = cos.shape[1]
    y = x.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = float(cos[position, i]), float(sin[position, i])
        y[a], y[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return y


def worth(score, position, seen, sinks, recent):
    """Ranks of the slots of one head, the first to be kept lowest: python's sort is stable, so equals stay in slot order."""
    def key(j):
        if position[j] < sinks or position[j] >= seen - recent:
            return (0, 0.0)
        return (2, 0.0) if math.isnan(score[j]) else (1, -score[j])
    return sorted(range(len(score)), key=key)


def plan(c, budget, sinks, recent):
    """moves by (sequence, head) as lists of (source, target), and the new lengths."""
    moves = {}
    seen = (c.seen if c.seen is not None else c.lengths).tolist()
    for s, length in enumerate(c.lengths.tolist()):
        pg, pl = places(c, s, length)
        for h in range(c.kv_heads):
            moves[s, h] = []
            if length <= budget:
                continue
            score = c.scores[pg, h, pl].tolist()
            position = c.positions[pg, h, pl].tolist() if c.positions is not None else list(range(length))
            kept = set(worth(score, position, seen[s], sinks, recent)[:budget])
            movers = [j for j in range(budget, length) if j in kept]
            holes = [j for j in range(budget) if j not in kept]
            assert len(movers) == len(holes)
            moves[s, h] = list(zip(movers, holes))
    return moves, [min(n, budget) for n in c.lengths.tolist()]


def evict(c, moves):
    for (s, h), pairs in moves.items():
        for source, target in pairs:
            a, b = ((int(c.table[s, j // c.page_size]), j % c.page_size) for j in (source, target))
            for x in (c.k, c.v):
                x[b[0], b[1], h] = x[a[0], a[1], h]
            for x in (c.scores, c.positions):
                if x is not None:
                    x[b[0], h, b[1]] = x[a[0], h, a[1]]
