"""The work on a key-value cache that is kept within a memory budget, as cases to be timed.

A program that serves a language model under a budget does this with the paged cache of every layer: it appends the keys and values of
the new tokens (`append`: norms per head, position rotation and the write to the pages in one pass), lets the new tokens' queries read
the cache and book the weight that each cached token received (`attend`), plans which tokens leave once a sequence is over its budget
(`plan`), and moves those that stay into the room of those that leave (`evict`).

Lengths follow from the case alone, contents and the pages' places from the seed.  Entries of the page table behind a sequence are -1.
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one user, a short conversation, as many key-value heads as query heads (16 heads of 64): latency is what counts
        dict(name="attend_one", do="attend", type="fp16", seqs=1, new=1, heads=16, kv=16, dim=64, longest=517, page=16, window=0, sinks=0, book=False, ragged=False),
        # a batch in the middle of its answers, the cache under a budget: weights are booked for the next eviction
        dict(name="attend_batch", do="attend", type="bf16", seqs=24, new=1, heads=32, kv=8, dim=128, longest=4100, page=16, window=0, sinks=0, book=True, ragged=False),
        # one very long document, before its first eviction
        dict(name="attend_long", do="attend", type="bf16", seqs=1, new=1, heads=32, kv=4, dim=128, longest=200003, page=64, window=0, sinks=0, book=True, ragged=False),
        # a full server: the largest call
        dict(name="attend_server", do="attend", type="bf16", seqs=64, new=1, heads=64, kv=8, dim=128, longest=16000, page=32, window=0, sinks=0, book=False, ragged=False),
        # layers with a sliding window that keep the first tokens visible, 16 heads of 80, pages of no power of two
        dict(name="attend_window", do="attend", type="fp16", seqs=16, new=1, heads=16, kv=16, dim=80, longest=30001, page=48, window=2047, sinks=5, book=False, ragged=False),
        # the last tokens of prompts (or drafts to be verified) looked at together, fewer of them in some sequences
        dict(name="attend_several", do="attend", type="bf16", seqs=6, new=16, heads=32, kv=8, dim=128, longest=9001, page=16, window=0, sinks=0, book=True, ragged=True),
        # the next token of a batch: norms, rotation, write
        dict(name="append_step", do="append", type="bf16", seqs=96, new=1, heads=32, kv=8, dim=128, longest=1000, page=16, rotary=128, interleaved=False, norm=True, ragged=False),
        # prompts of odd lengths, half of each head rotated in interleaved pairs
        dict(name="append_prompt", do="append", type="fp16", seqs=3, new=4097, heads=16, kv=16, dim=64, longest=4500, page=32, rotary=32, interleaved=True, norm=True, ragged=True),
        # a batch that is over its budget by the tokens of the last turns
        dict(name="plan_step", do="plan", seqs=32, kv=8, longest=2112, page=16, budget=2048, sinks=4, recent=64),
        # long prompts brought down to the budget
        dict(name="plan_prompt", do="plan", seqs=2, kv=8, longest=65537, page=64, budget=4096, sinks=4, recent=256),
        # what those two plans move
        dict(name="evict_step", do="evict", type="bf16", dim=128, seqs=32, kv=8, longest=2112, page=16, budget=2048, sinks=4, recent=64),
        dict(name="evict_prompt", do="evict", type="fp16", dim=128, seqs=2, kv=8, longest=65537, page=64, budget=4096, sinks=4, recent=256),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(("attend", "attend", "attend", "append", "plan", "evict"))
    kind = rng.choice(("bf16", "bf16", "fp16"))
    dim = rng.choice((64, 64, 80, 96, 128, 128, 128, 192, 256))
    kv = rng.choice((1, 2, 4, 8, 8, 16))
    group = rng.choice((1, 1, 2, 3, 4, 4, 5, 7, 8, 16))
    page = rng.choice((1, 8, 16, 16, 24, 32, 64, 100, 128))
    seqs = _spread(rng, 1, 64)
    if do == "attend":
        new = rng.choice((1, 1, 1, 2, 5, 16))
        room = 60_000_000 // (kv * dim * (new * group if new > 1 else 1))      # (tokens of all sequences)
        longest = max(new, _spread(rng, 1, max(2, min(150000, 8 * room // seqs))))
        window = rng.choice((0, 0, _spread(rng, 16, 5000)))
        return dict(do=do, type=kind, seqs=seqs, new=new, heads=kv * group, kv=kv, dim=dim, longest=longest, page=page, window=window,
                    sinks=rng.choice((0, 1, 4, 17)) if window else 0, book=rng.random() < 0.5, ragged=new > 1 and rng.random() < 0.5)
    if do == "append":
        new = rng.choice((1, _spread(rng, 2, 4000)))
        seqs = min(seqs, max(1, 12000 // new))
        rotary = rng.choice((0, dim, dim, dim // 2))
        return dict(do=do, type=kind, seqs=seqs, new=new, heads=kv * group, kv=kv, dim=dim, longest=new + _spread(rng, 1, 2000), page=page,
                    rotary=rotary, interleaved=rotary > 0 and rng.random() < 0.4, norm=rng.random() < 0.7, ragged=new > 1 and rng.random() < 0.5)
    budget = _spread(rng, 32, 8000)
    longest = min(max(budget + 1, int(budget * math.exp(rng.uniform(0.0, 3.0)))), 8_000_000 // (seqs * kv) + budget)
    case = dict(seqs=seqs, kv=kv, longest=longest, page=page, budget=budget, sinks=rng.choice((0, 1, 4)), recent=rng.choice((0, 1, budget // 8, budget // 2)))
    return dict(do="plan", **case) if do == "plan" else dict(do="evict", type=kind, dim=min(dim, 128), **case)


# ---- sizes of a case -------------------------------------------------------------------------------------------------
def _lengths(case):
    """Tokens in each sequence: the first is the longest, the others lie between a fifth of it and itself (near the longest where a
    budget is exceeded by a little)."""
    most, least = case["longest"], max(1, case["longest"] // 5, case.get("new", 1))
    if case["do"] in ("plan", "evict"):
        least = max(1, case["budget"] - (most - case["budget"]) // 4)
    return [most if i == 0 else least + int((most - least) * ((i * 0.6180339887) % 1.0)) for i in range(case["seqs"])]


def _counts(case):
    """New tokens of each sequence, at most case["new"]."""
    n = case["new"]
    return [n if not case["ragged"] or i % 3 == 0 else 1 + (7 * i) % n for i in range(case["seqs"])]


def _visible(case):
    """Slots that some row of the sequence sees, for each sequence."""
    if not case["window"]:
        return _lengths(case)
    seen = []
    for length, count in zip(_lengths(case), _counts(case)):
        first = max(0, length - count - case["window"] + 1)
        seen.append(length - first + min(first, case["sinks"]))
    return seen


# ---- a user's program ------------------------------------------------------------------------------------------------
def _metadata(case, gen):
    """Lengths, and a page table whose pages lie anywhere in the pool, with a few pages that nobody has."""
    lengths = _lengths(case)
    page = case["page"]
    columns = -(-case["longest"] // page)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device=DEV).int()
    first = torch.tensor([0] + need, device=DEV).cumsum(0)
    at = torch.arange(columns, device=DEV)
    table = torch.where(at[None] < torch.tensor(need, device=DEV)[:, None], order[(first[:-1, None] + at[None]).clamp(max=pages - 1)], -1).int()
    return dict(lengths=torch.tensor(lengths, device=DEV, dtype=torch.int32), table=table, pages=pages, page=page, longest=case["longest"], spare=order[-1].long())


def _scores(case, pages, gen):
    """Accumulated weights: most tokens get little, a few get much, some none at all."""
    s = torch.exp(2.0 * torch.randn(pages, case["kv"], case["page"], generator=gen, device=DEV)) * 0.01
    return s * (torch.rand(s.shape, generator=gen, device=DEV) > 0.05)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case, **_metadata(case, gen))
    do, kv = case["do"], case["kv"]
    if do in ("plan", "evict"):
        s["scores"] = _scores(case, s["pages"], gen)
        # (a cache that was evicted before: each head has its tokens in an order of its own)
        s["seen"] = s["lengths"] + 1000
        s["positions"] = _positions(s, gen)
        moves = (case["seqs"], kv, case["budget"], 2)
        if do == "plan":
            s["out"] = dict(moves=torch.full(moves, -1, dtype=torch.int32, device=DEV), counts=torch.zeros(moves[:2], dtype=torch.int32, device=DEV),
                            lengths=torch.zeros(case["seqs"], dtype=torch.int32, device=DEV))
            return s
        s["moves"], s["counts"], _ = _plain_plan(s)
    dtype = TYPES[case["type"]]
    normal = lambda *shape: torch.randn(shape, generator=gen, device=DEV, dtype=dtype)
    dim = case["dim"]
    s["k"], s["v"] = normal(s["pages"], s["page"], kv, dim), normal(s["pages"], s["page"], kv, dim)
    if do == "evict":
        return s
    seqs, new, heads = case["seqs"], case["new"], case["heads"]
    s["count"] = torch.tensor(_counts(case), device=DEV, dtype=torch.int32) if case["ragged"] else None
    if do == "attend":
        s["q"] = 2.0 * normal(seqs, new, heads, dim)
        s["scale"] = 1.0 / math.sqrt(dim)
        s["scores"] = _scores(case, s["pages"], gen) if case["book"] else None
        s["out"] = torch.zeros(seqs, new, heads, dim, device=DEV, dtype=dtype)
        s["lse"] = torch.zeros(seqs, new, heads, device=DEV)
        return s
    # one projection's output holds queries, keys and values side by side
    both = normal(seqs, new, heads + 2 * kv, dim)
    s["new_q"], s["new_k"], s["new_v"] = both[:, :, :heads], both[:, :, heads:heads + kv], both[:, :, heads + kv:]
    s["scores"] = _scores(case, s["pages"], gen)
    s["positions"] = torch.zeros(s["scores"].shape, dtype=torch.int32, device=DEV)
    s["q_weight"] = 1.0 + 0.1 * normal(dim) if case["norm"] else None
    s["k_weight"] = 1.0 + 0.1 * normal(dim) if case["norm"] else None
    s["cos"] = s["sin"] = None
    if case["rotary"]:
        half = case["rotary"] // 2
        angle = torch.arange(case["longest"], device=DEV, dtype=torch.float64)[:, None] * torch.pow(
            10000.0, -torch.arange(half, device=DEV, dtype=torch.float64) / half)[None]
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    s["out"] = torch.zeros(seqs, new, heads, dim, device=DEV, dtype=dtype)
    return s


def _handle(s):
    """The program's view of its cache, made once."""
    from paper_2310_09443_b200 import binding as g10
    if "handle" not in s:
        s["handle"] = g10.CacheBuffers(s.get("k"), s.get("v"), s["table"], s["lengths"], seen=s.get("seen"), scores=s.get("scores"),
                                       positions=s.get("positions"), page_size=s["page"], kv_heads=s["kv"])
    return g10, s["handle"]


def run(s):
    do = s["do"]
    if not own:
        return {"attend": _plain_attend, "append": _plain_append, "plan": _plain_planned, "evict": _plain_evict}[do](s)
    g10, cache = _handle(s)
    if do == "attend":
        if "ws" not in s:
            s["ws"] = torch.empty(g10.g10_cache_workspace_bytes(cache, s["new"], s["heads"], add_scores=s["book"]), dtype=torch.uint8, device=DEV)
        g10.g10_cache_attend(cache, s["q"], scale=s["scale"], window=s["window"], sinks=s["sinks"], counts=s["count"], add_scores=s["book"],
                             out=s["out"], lse=s["lse"], ws=s["ws"])
        return _attended(s, s["out"], s["lse"])
    if do == "append":
        g10.g10_cache_append(cache, s["new_k"], s["new_v"], s["new_q"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6, cos=s["cos"],
                             sin=s["sin"], interleaved=s["interleaved"], counts=s["count"], q_out=s["out"])
        return _appended(s, s["out"])
    if do == "plan":
        o = s["out"]
        g10.g10_cache_plan_evictions(cache, s["budget"], sinks=s["sinks"], recent=s["recent"], moves=o["moves"], counts=o["counts"], new_lengths=o["lengths"])
        return o
    g10.g10_cache_evict(cache, s["moves"], s["counts"])
    return _evicted(s)


def _attended(s, out, lse):
    return dict(out=out, lse=lse, scores=s["scores"]) if s["book"] else dict(out=out, lse=lse)


def _appended(s, q):
    return dict(q=q, k=s["k"], v=s["v"], scores=s["scores"], positions=s["positions"])


def _evicted(s):
    return dict(k=s["k"], v=s["v"], scores=s["scores"], positions=s["positions"])


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _places(s):
    """Page and place in the page of every slot up to the longest sequence, and whether the sequence has the slot: [seqs, slots]."""
    at = torch.arange(s["longest"], device=DEV)
    return s["table"].long()[:, at // s["page"]].clamp(min=0), (at % s["page"]).expand(s["table"].shape[0], -1), at[None] < s["lengths"][:, None]


def _plain_attend(s):
    page, place, there = _places(s)
    seqs, new, heads, dim = s["q"].shape
    kv = s["kv"]
    k, v = (torch.where(there[:, :, None, None], s[x][page, place].float(), 0.0) for x in ("k", "v"))
    q = s["q"].float().view(seqs, new, kv, heads // kv, dim)
    count = s["count"] if s["count"] is not None else torch.full_like(s["lengths"], new)
    token = torch.arange(new, device=DEV)
    slot = (s["lengths"] - count)[:, None] + token[None]                      # [seqs, new]
    at = torch.arange(s["longest"], device=DEV)
    sees = (at <= slot[:, :, None]) & (token[None] < count[:, None])[:, :, None] & there[:, None]
    if s["window"]:
        sees &= (at < s["sinks"]) | (at > slot[:, :, None] - s["window"])
    score = torch.einsum("bnkgd,bckd->bkgnc", q, k) * s["scale"]
    score = torch.where(sees[:, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = weight.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    weight = weight / torch.where(total == 0.0, 1.0, total)
    out = torch.einsum("bkgnc,bckd->bnkgd", weight, v).reshape(seqs, new, heads, dim).to(s["q"].dtype)
    if s["book"]:
        head = torch.arange(kv, device=DEV)
        s["scores"].index_put_((page[:, :, None], head[None, None], place[:, :, None]), weight.sum((2, 3)).transpose(1, 2), accumulate=True)
    return _attended(s, out, lse.permute(0, 3, 1, 2).reshape(seqs, new, heads))


def _plain_turn(x, weight, cos, sin, interleaved):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.float()
    if cos is None:
        return x
    half = cos.shape[-1]
    cos, sin = cos[:, :, None], sin[:, :, None]
    turned, rest = x[..., :2 * half], x[..., 2 * half:]
    if interleaved:
        a, b = turned[..., 0::2], turned[..., 1::2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)
    a, b = turned[..., :half], turned[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)


def _plain_append(s):
    seqs, new = s["new_q"].shape[:2]
    count = s["count"] if s["count"] is not None else torch.full_like(s["lengths"], new)
    token = torch.arange(new, device=DEV)[None]
    there = token < count[:, None]
    slot = torch.where(there, (s["lengths"] - count)[:, None] + token, 0)
    # a token that does not count writes what is there already to a page that nobody has
    page = torch.where(there, s["table"].long().gather(1, (slot // s["page"]).long()), s["spare"])
    place = (slot % s["page"]).long()
    cos, sin = (None, None) if s["cos"] is None else (s["cos"][slot], s["sin"][slot])
    turn = lambda x, weight: _plain_turn(x, weight, cos, sin, s["interleaved"]).to(x.dtype)
    wide = there[:, :, None, None]
    q = torch.where(wide, turn(s["new_q"], s["q_weight"]), 0.0)
    s["k"][page, place] = torch.where(wide, turn(s["new_k"], s["k_weight"]), s["k"][page, place])
    s["v"][page, place] = torch.where(wide, s["new_v"], s["v"][page, place])
    s["scores"][page, :, place] = torch.where(there[:, :, None], 0.0, s["scores"][page, :, place])
    s["positions"][page, :, place] = torch.where(there[:, :, None], slot[:, :, None].int(), s["positions"][page, :, place])
    return _appended(s, q)


def _positions(s, gen):
    """Positions of the tokens that a cache evicted before holds: as many of the tokens seen as it has slots, in any order."""
    page, place, there = _places(s)
    kv = s["kv"]
    slots = s["longest"]
    mixed = torch.rand(there.shape[0], kv, slots, generator=gen, device=DEV) + (~there[:, None]).float()
    rank = mixed.argsort(-1).argsort(-1).int()                                # [seqs, kv, slots]: 0 .. length - 1 where there is a token
    position = torch.where(rank < 500, rank, rank + 1000)
    out = torch.full((s["pages"], kv, s["page"]), -1, dtype=torch.int32, device=DEV)
    cell = (page[:, :, None].expand(-1, -1, kv)[there], torch.arange(kv, device=DEV).expand(there.shape + (kv,))[there], place[:, :, None].expand(-1, -1, kv)[there])
    out[cell] = position.transpose(1, 2)[there]
    return out


def _plain_plan(s):
    page, place, there = _places(s)
    kv, budget = s["kv"], s["budget"]
    head = torch.arange(kv, device=DEV)[None, None]
    cell = (page[:, :, None], head, place[:, :, None])
    score, position = s["scores"][cell].transpose(1, 2), s["positions"][cell].transpose(1, 2)   # [seqs, kv, slots]
    there = there[:, None]
    stays = (position < s["sinks"]) | (position >= (s["seen"] - s["recent"])[:, None, None])
    worth = torch.where(there, torch.where(stays, math.inf, score), -math.inf)
    rank = torch.sort(worth, dim=-1, descending=True, stable=True).indices.argsort(-1)
    kept = (rank < budget) & there
    at = torch.arange(s["longest"], device=DEV).expand_as(kept)
    over = (s["lengths"] > budget)[:, None, None]
    mover, hole = kept & (at >= budget) & over, ~kept & (at < budget) & over
    moves = torch.full(kept.shape[:2] + (budget + 1, 2), -1, dtype=torch.int32, device=DEV)
    for which, side in ((mover, 0), (hole, 1)):                                # (the last entry takes what is neither)
        nth = torch.where(which, which.cumsum(-1) - 1, budget)
        moves[..., side].scatter_(-1, nth, torch.where(which, at, -1).int())
    return moves[:, :, :budget].contiguous(), mover.sum(-1).int(), s["lengths"].clamp(max=budget)


def _plain_planned(s):
    moves, counts, lengths = _plain_plan(s)
    return dict(moves=moves, counts=counts, lengths=lengths)


def _plain_evict(s):
    kv, budget = s["kv"], s["budget"]
    real = torch.arange(budget, device=DEV) < s["counts"][:, :, None]
    seq = torch.arange(s["table"].shape[0], device=DEV)[:, None, None]
    head = torch.arange(kv, device=DEV)[None, :, None].expand_as(real)
    # (an entry that is no move copies the first slot onto itself)
    source, target = (torch.where(real, s["moves"][..., side], 0).long() for side in (0, 1))
    found = s["table"].long()
    pages = [found[seq, x // s["page"]] for x in (source, target)]
    places = [x % s["page"] for x in (source, target)]
    same = ~real & (s["counts"] > 0)[:, :, None]
    # (the first slot may be a hole: such an entry repeats the sequence's first move instead)
    pages = [torch.where(same, p[:, :, :1], p) for p in pages]
    places = [torch.where(same, p[:, :, :1], p) for p in places]
    for pool in (s["k"], s["v"]):
        pool[pages[1], places[1], head] = pool[pages[0], places[0], head]
    for table in (s["scores"], s["positions"]):
        table[pages[1], head, places[1]] = table[pages[0], head, places[0]]
    return _evicted(s)


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    do = case["do"]
    if do == "plan":
        return None                                                           # (whole numbers)
    lengths, table, page = s["lengths"].tolist(), s["table"].tolist(), s["page"]
    pick = lambda b, n: (torch.tensor(table[b], device=DEV).repeat_interleave(page)[:n].long(), torch.arange(n, device=DEV) % page)
    if do == "evict":
        k, v, scores = s["k"].double(), s["v"].double(), s["scores"].double()
        moves, counts = s["moves"].cpu(), s["counts"].tolist()
        for b in range(case["seqs"]):
            pages, places = pick(b, lengths[b])
            for h in range(case["kv"]):
                source, target = moves[b, h, :counts[b][h]].long().to(DEV).T
                for pool in (k, v):
                    pool[pages[target], places[target], h] = pool[pages[source], places[source], h]
                scores[pages[target], h, places[target]] = scores[pages[source], h, places[source]]
        return dict(k=k, v=v, scores=scores, positions=None)
    counts = _counts(case)
    group = case["heads"] // case["kv"]
    if do == "append":
        k, v, scores = s["k"].double(), s["v"].double(), s["scores"].double()
        q = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
        half = case["rotary"] // 2
        first = torch.arange(half, device=DEV) * (2 if case["interleaved"] else 1)
        second = first + (1 if case["interleaved"] else half)

        def turned(x, weight, slots):
            x = x.double()
            if weight is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * weight.double()
            if not half:
                return x
            z = torch.complex(x[..., first], x[..., second]) * torch.complex(s["cos"].double(), s["sin"].double())[slots][:, None]
            y = x.clone()
            y[..., first], y[..., second] = z.real, z.imag
            return y

        for b, (length, count) in enumerate(zip(lengths, counts)):
            pages, places = (x[length - count:] for x in pick(b, length))
            slots = torch.arange(length - count, length, device=DEV)
            q[b, :count] = turned(s["new_q"][b, :count], s["q_weight"], slots)
            k[pages, places] = turned(s["new_k"][b, :count], s["k_weight"], slots)
            v[pages, places] = s["new_v"][b, :count].double()
            scores[pages, :, places] = 0.0
        return dict(q=q, k=k, v=v, scores=scores, positions=None)
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    scores = s["scores"].double() if case["book"] else None
    for b, (length, count) in enumerate(zip(lengths, counts)):
        pages, places = pick(b, length)
        slot = torch.arange(length, device=DEV)
        for h in range(case["kv"]):
            k, v = s["k"][pages, places, h].double(), s["v"][pages, places, h].double()
            mine = slice(h * group, (h + 1) * group)
            for t in range(count):
                p = length - count + t
                sees = slot <= p
                if case["window"]:
                    sees = sees & ((slot < case["sinks"]) | (slot > p - case["window"]))
                logit = (s["q"][b, t, mine].double() @ k.T * s["scale"]).masked_fill(~sees, -math.inf)
                lse[b, t, mine] = logit.logsumexp(-1)
                weight = (logit - lse[b, t, mine, None]).exp()
                out[b, t, mine] = weight @ v
                if scores is not None:
                    scores[pages, h, places] += weight.sum(0)
    return dict(out=out, lse=lse, scores=scores) if case["book"] else dict(out=out, lse=lse)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def work(case):
    """Each row of keys and values that is visible read once (attend), each new token read and written once (append), scores and positions
    of the sequences over their budget read once (plan), each moved row read and written once (evict; the share of the kept
    tokens that stand behind the budget is that of all)."""
    do, kv, lengths = case["do"], case["kv"], _lengths(case)
    if do == "attend":
        rows = case["new"] * case["heads"]
        slots = sum(_visible(case))
        n = slots * kv * case["dim"] * 4 + case["seqs"] * rows * (case["dim"] * 4 + 4) + (8 * slots * kv if case["book"] else 0)
        return {"bytes": n, "flops": 4 * sum(v * c for v, c in zip(_visible(case), _counts(case))) * case["heads"] * case["dim"]}
    if do == "append":
        tokens = sum(_counts(case))
        return {"bytes": tokens * (case["heads"] + 2 * kv) * case["dim"] * 4 + tokens * (8 * kv + 4 * case["rotary"]),
                "flops": tokens * (case["heads"] + kv) * case["dim"] * 7}
    over = [n for n in lengths if n > case["budget"]]
    moves = sum(case["budget"] * (n - case["budget"]) // n for n in over) * kv
    if do == "plan":
        return {"bytes": 8 * sum(over) * kv + 8 * moves, "flops": 0}
    return {"bytes": moves * (case["dim"] * 8 + 24), "flops": 0}
