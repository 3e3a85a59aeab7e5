"""Rows of 8-bit codes restated in 64 bits, and caches of them for tests (on top of cache_oracle.py)."""
import math

import torch

import cache_oracle as O

CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
LARGEST = {"int8": 127.0, "e4m3": 448.0}


def nearest(x, code):
    """The nearest value that a code stands for (64 bits, in units of the scale), ties to even."""
    if code == "int8":
        return x.round()
    unit = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)      # (below 2^-6 steps of 2^-9)
    return (x / unit).round() * unit


def step_of(x, code):
    """Distance of neighbouring codes' values about x."""
    return torch.ones_like(x) if code == "int8" else torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)


def packed(x, code):
    """Codes and scales (32 bits) of rows x [.., dim] in 64 bits."""
    top = x.abs().amax(-1, keepdim=True)
    scale = top / LARGEST[code]
    y = nearest(torch.where(top > 0, x / torch.where(top > 0, scale, 1.0), 0.0), code)
    return y.to(torch.int8) if code == "int8" else y.float().to(torch.float8_e4m3fn), scale.squeeze(-1).float()


def make_packed(lengths, kv_heads, head_dim, page_size, dtype, code, seed, spread=0.5, garbage=True, **more):
    """A cache of packed rows on the host.  Where no token stands: codes of any kind (no number in e4m3), scales that are none.  c.k and c.v are the values that the
    codes stand for, in 64 bits."""
    c = O.make_cache(lengths, kv_heads, head_dim, page_size, dtype, seed, garbage=False, **more)
    gen = torch.Generator().manual_seed(seed + 5)
    owned = torch.zeros(c.k.shape[:2], dtype=torch.bool)
    for s, n in enumerate(lengths):
        pg, pl = O.places(c, s, n)
        owned[pg, pl] = True
    c.code, c.owned = code, owned
    sides = []
    for x in (c.k, c.v):
        x = x.double() * torch.exp(spread * torch.randn(x.shape[:3], generator=gen).double())[..., None]
        codes, scale = packed(x, code)
        if garbage:
            bad = torch.randint(-128, 128, x.shape, generator=gen, dtype=torch.int8)
            if code == "e4m3":
                bad = torch.where(torch.rand(x.shape, generator=gen) < 0.5, torch.tensor(127, dtype=torch.int8), bad).view(torch.float8_e4m3fn)
            codes.view(torch.int8)[~owned] = bad.view(torch.int8)[~owned]
            scale[~owned] = math.nan
        sides.append((codes, scale))
    (c.kc, ks), (c.vc, vs) = sides
    c.scales = torch.stack([ks, vs], -1).transpose(1, 2).contiguous()
    values(c)
    return c


def values(c):
    """c.k and c.v from codes and scales."""
    c.k, c.v = (codes.double() * c.scales[..., side].transpose(1, 2).double()[..., None] for side, codes in ((0, c.kc), (1, c.vc)))


def rounded(c):
    """c.k and c.v as they are read back."""
    c.k, c.v = c.k.to(c.dtype), c.v.to(c.dtype)


def upload(g10, c, device="cuda:0", **more):
    def rows(x):
        if c.layout == "heads":
            return x.view(torch.int8).transpose(1, 2).contiguous().to(device).transpose(1, 2).view(x.dtype)
        if c.layout == "wide":                         # rows of a larger tensor
            big = torch.full((x.shape[0], 2, x.shape[1], x.shape[2], x.shape[3] + 16), 127, dtype=torch.int8, device=device)
            big[:, 1, :, :, 16:] = x.view(torch.int8).to(device)
            return big[:, 1, :, :, 16:].view(x.dtype)
        return x.to(device)
    on = lambda x: None if x is None else x.to(device)
    return g10.PackedBuffers(rows(c.kc), rows(c.vc), on(c.scales), on(c.table), on(c.lengths), dtype=c.dtype, seen=on(c.seen), scores=on(c.scores),
                             positions=on(c.positions), **more)


def attend_bounds(c, r, q, scale):
    """How far out, lse and a weight (relatively) may be off: attend_bounds of cache_oracle.py, with these differences.

    int8 keys are multiplied 128 too large, and 128 times the sum of the queries is taken off: D more additions, and terms of size (|code| + 128) ks |q|.  bf16 queries lose
    what is below 2^-39 of the row's largest element: far less than one of the units counted.  Weights times the value's scale are rounded to fp16: half a step relative, or 2^-25
    where the largest of the row (for more than 16 rows its largest weight times the largest scale, or half of that) is at least 2^10.  They come from a logarithm of the scale
    off by 2^-22 relatively or absolutely, and an addition; or from two products more."""
    seqs, new, heads, dim = q.shape
    group = heads // c.kv_heads
    step = O.half_step(c.dtype)
    slip, tiny = r.slip.clone(), torch.zeros_like(r.out)
    logs = torch.zeros_like(r.slip)
    for s, n in enumerate(c.lengths.tolist()):
        if n == 0:
            continue
        pg, pl = O.places(c, s, n)
        for h in range(c.kv_heads):
            mine = slice(h * group, (h + 1) * group)
            ks, vs = (c.scales[pg, h, pl, side].double() for side in (0, 1))
            if c.code == "int8":
                slip[s, :, mine] += 128 * ks.max() * q[s, :, mine].double().abs().sum(-1) * abs(scale)
            logs[s, :, mine] = (torch.log2(vs.clamp(min=2.0 ** -126)).abs()).max()
            tiny[s, :, mine] = 2.0 ** -34 * vs.max() * c.vc[pg, pl, h].double().abs().sum(0)
    d = (2 * dim + 8) * 2.0 ** -23 * slip
    rel = 2 * d + 2.0 ** -21 + (r.n_seen + 8) * 2.0 ** -23 + 2.0 ** -22 * (logs + 1)
    out = (2.0 ** -11 + rel[..., None] + (r.n_seen[..., None] + 8) * 2.0 ** -23) * r.weighed * 1.01 + tiny
    out = out + step * (r.out.abs() + out) + (2.0 ** -25 if c.dtype == torch.float16 else 0.0)
    return out, d + rel + 2.0 ** -22 * r.lse.abs(), rel


def evict(c, moves):
    """cache_oracle's on codes and scales."""
    c.k, c.v = c.kc.view(torch.int8), c.vc.view(torch.int8)
    O.evict(c, moves)
    for (s, h), pairs in moves.items():
        for source, target in pairs:
            a, b = ((int(c.table[s, j // c.page_size]), j % c.page_size) for j in (source, target))
            c.scales[b[0], h, b[1]] = c.scales[a[0], h, a[1]]
    values(c)
