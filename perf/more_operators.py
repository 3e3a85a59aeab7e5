"""More work on a key-value cache that is kept within a memory budget, as cases to be timed.

A program that serves a language model has two more ways to make room for tokens.  It keeps rows in 8 bits: new tokens are quantised as they
are written, each row of a head with a scale of its own (`write`, which reads the new rows back as well: what the codes stand for), prompts are read
back (`read`), the new tokens' queries attend the packed rows as they are (`attend`), and rows move with their scales when a sequence is over
its budget (`evict`).  And sequences that begin alike share the pages of their beginning, which one pass over it then serves for all of
them (`shared`).

Lengths follow from the case alone, contents and the pages' places from the seed.  Entries of the page table behind a sequence are -1.
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
LARGEST = {"int8": 127.0, "e4m3": 448.0}


def listed():
    return [
        # the next token of a batch: norms, rotation, quantised and written
        dict(name="write_step", do="write", type="bf16", code="int8", seqs=96, new=1, heads=32, kv=8, dim=128, longest=1000, page=16, rotary=128, interleaved=False, norm=True, ragged=False),
        # prompts of odd lengths, half of each head rotated in interleaved pairs
        dict(name="write_prompt", do="write", type="fp16", code="e4m3", seqs=3, new=4097, heads=16, kv=16, dim=64, longest=4500, page=32, rotary=32, interleaved=True, norm=True, ragged=True),
        # the last tokens of a batch, for a program that looks at them again
        dict(name="read_batch", do="read", type="fp16", code="e4m3", seqs=24, kv=16, dim=80, longest=2100, page=24, tokens=333, tail=True),
        # a long prompt and a shorter one, read back whole to be attended in parts with many rows
        dict(name="read_prompt", do="read", type="bf16", code="int8", seqs=2, kv=8, dim=128, longest=65537, page=64, tokens=65537, tail=False),
        # one user, a short conversation, as many key-value heads as query heads: latency is what counts
        dict(name="attend_one", do="attend", type="fp16", code="e4m3", seqs=1, new=1, heads=16, kv=16, dim=64, longest=517, page=16, window=0, sinks=0, book=False, ragged=False),
        # a batch in the middle of its answers, the cache under a budget: weights are booked for the next eviction
        dict(name="attend_batch", do="attend", type="bf16", code="int8", seqs=24, new=1, heads=32, kv=8, dim=128, longest=4100, page=16, window=0, sinks=0, book=True, ragged=False),
        # a full server: the largest call
        dict(name="attend_server", do="attend", type="bf16", code="e4m3", seqs=64, new=1, heads=64, kv=8, dim=128, longest=16000, page=32, window=0, sinks=0, book=False, ragged=False),
        # what the plan for a batch that is over its budget by the tokens of the last turns moves
        dict(name="evict_step", do="evict", code="int8", dim=128, seqs=32, kv=8, longest=2112, page=16, budget=2048, sinks=4, recent=64),
        # long prompts brought down to the budget
        dict(name="evict_prompt", do="evict", code="e4m3", dim=128, seqs=2, kv=8, longest=65537, page=64, budget=4096, sinks=4, recent=256),
        # four answers to one question of some hundred tokens
        dict(name="shared_few", do="shared", type="fp16", seqs=4, new=1, heads=16, kv=16, dim=64, prefix=1000, own=61, page=16, ragged=False),
        # a long document that many ask about: the answers are short beside it
        dict(name="shared_server", do="shared", type="bf16", seqs=64, new=1, heads=64, kv=8, dim=128, prefix=32000, own=1500, page=32, ragged=False),
        # drafts of several tokens, verified for a batch behind the same instructions; heads of 96, pages of no power of two
        dict(name="shared_drafts", do="shared", type="bf16", seqs=23, new=7, heads=24, kv=6, dim=96, prefix=6010, own=700, page=24, ragged=True),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(("write", "read", "attend", "attend", "attend", "evict", "shared", "shared", "shared"))
    kind, code = rng.choice(("bf16", "bf16", "fp16")), rng.choice(("int8", "e4m3"))
    dim = rng.choice((64, 64, 80, 96, 112, 128, 128, 128, 192, 256))
    kv = rng.choice((1, 2, 4, 8, 8, 16))
    group = rng.choice((1, 1, 2, 3, 4, 4, 5, 7, 8, 16))
    page = rng.choice((1, 8, 16, 16, 24, 32, 64, 100, 128))
    seqs = _spread(rng, 1, 64)
    if do == "attend":
        new = rng.choice((1, 1, 1, 1, 2, 5, 16))
        room = 60_000_000 // (kv * dim * (new * group if new > 1 else 1))      # (tokens of all sequences)
        longest = max(new, _spread(rng, 1, max(2, min(150000, 8 * room // seqs))))
        window = rng.choice((0, 0, _spread(rng, 16, 5000)))
        return dict(do=do, type=kind, code=code, seqs=seqs, new=new, heads=kv * group, kv=kv, dim=dim, longest=longest, page=page, window=window,
                    sinks=rng.choice((0, 1, 4, 17)) if window else 0, book=rng.random() < 0.5, ragged=new > 1 and rng.random() < 0.5)
    if do == "write":
        new = rng.choice((1, _spread(rng, 2, 4000)))
        seqs = min(seqs, max(1, 12000 // new))
        rotary = rng.choice((0, dim, dim, dim // 2))
        return dict(do=do, type=kind, code=code, seqs=seqs, new=new, heads=kv * group, kv=kv, dim=dim, longest=new + _spread(rng, 1, 2000), page=page,
                    rotary=rotary, interleaved=rotary > 0 and rng.random() < 0.4, norm=rng.random() < 0.7, ragged=new > 1 and rng.random() < 0.5)
    if do == "read":
        longest = _spread(rng, 1, min(150000, max(2, 100_000_000 // (seqs * kv * dim))))
        return dict(do=do, type=kind, code=code, seqs=seqs, kv=kv, dim=dim, longest=longest, page=page, tokens=rng.choice((longest, _spread(rng, 1, max(2, longest)))),
                    tail=rng.random() < 0.5)
    if do == "shared":
        new = rng.choice((1, 1, 1, 2, 5, 16))
        rows = new * group
        behind = max(new, _spread(rng, 1, 3000), 1)
        prefix = _spread(rng, 64, max(65, min(150000, 60_000_000_000 // (seqs * rows * kv * dim) // 8)))
        return dict(do=do, type=kind, seqs=seqs, new=new, heads=kv * group, kv=kv, dim=dim, prefix=prefix, own=min(behind, max(new, 100_000_000 // (seqs * rows * kv * 8))), page=page,
                    ragged=new > 1 and rng.random() < 0.5)
    budget = _spread(rng, 32, 8000)
    longest = min(max(budget + 1, int(budget * math.exp(rng.uniform(0.0, 3.0)))), 8_000_000 // (seqs * kv) + budget)
    return dict(do=do, code=code, dim=min(dim, 128), seqs=seqs, kv=kv, longest=longest, page=page, budget=budget, sinks=rng.choice((0, 1, 4)),
                recent=rng.choice((0, 1, budget // 8, budget // 2)))


# ---- sizes of a case -------------------------------------------------------------------------------------------------
def _common(case):
    """Slots that all sequences share: whole pages."""
    return case["prefix"] // case["page"] * case["page"] if case["do"] == "shared" else 0


def _lengths(case):
    """Tokens in each sequence: the first is the longest, the others lie between a fifth of it and itself (near the longest where a budget is
    exceeded by a little; behind the shared beginning, where there is one)."""
    most, before = case.get("longest", 0), 0
    if case["do"] == "shared":
        most, before = case["own"], case["prefix"]
    least = max(1, most // 5, case.get("new", 1))
    if case["do"] == "evict":
        least = max(1, case["budget"] - (most - case["budget"]) // 4)
    return [before + (most if i == 0 else least + int((most - least) * ((i * 0.6180339887) % 1.0))) for i in range(case["seqs"])]


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
    """Lengths, and a page table whose pages lie anywhere in the pool, with a few pages that nobody has; pages of a shared beginning are the same
    for all."""
    lengths, page, common = _lengths(case), case["page"], _common(case) // case["page"]
    columns = -(-max(lengths) // page)
    need = [-(-n // page) - common for n in lengths]
    pages = common + sum(need) + 3
    order = torch.randperm(pages, generator=gen, device=DEV).int()
    first = common + torch.tensor([0] + need, device=DEV).cumsum(0)
    at = torch.arange(columns, device=DEV)[None]
    its = order[(first[:-1, None] + at - common).clamp(min=0, max=pages - 1)]
    table = torch.where(at < common, order[at.clamp(max=pages - 1)], torch.where(at - common < torch.tensor(need, device=DEV)[:, None], its, -1)).int()
    return dict(lengths=torch.tensor(lengths, device=DEV, dtype=torch.int32), table=table.contiguous(), pages=pages, page=page, longest=max(lengths), spare=order[-1].long())


def _scores(case, pages, gen):
    """Accumulated weights: most tokens get little, a few get much, some none at all."""
    s = torch.exp(2.0 * torch.randn(pages, case["kv"], case["page"], generator=gen, device=DEV)) * 0.01
    return s * (torch.rand(s.shape, generator=gen, device=DEV) > 0.05)


def _quantised(x, code):
    """Codes and scales of rows x [.., dim] in 32 bits, from the definition: scale = largest / 127 (or 448), code = x * (127 / largest), rounded."""
    top = x.abs().amax(-1, keepdim=True)
    y = x * torch.where(top > 0.0, LARGEST[code] / top, 0.0)
    y = torch.round(y).to(torch.int8) if code == "int8" else y.to(torch.float8_e4m3fn)
    return y, (top / LARGEST[code]).squeeze(-1)


def _packed(case, pages, gen):
    """Rows that were written earlier, and their scales [pages, kv, page, 2]."""
    kv, page, dim = case["kv"], case["page"], case["dim"]
    dtype = CODES[case["code"]]
    codes = [torch.empty(pages, page, kv, dim, dtype=dtype, device=DEV) for _ in range(2)]
    scales = torch.empty(pages, kv, page, 2, device=DEV)
    step = max(1, 50_000_000 // (page * kv * dim))
    for i in range(0, pages, step):
        n = min(step, pages - i)
        for side in range(2):
            x = torch.randn(n, page, kv, dim, generator=gen, device=DEV) * torch.exp(0.5 * torch.randn(n, page, kv, 1, generator=gen, device=DEV))
            codes[side][i:i + n], s = _quantised(x, case["code"])
            scales[i:i + n, :, :, side] = s.transpose(1, 2)
    return codes[0], codes[1], scales


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case, **_metadata(case, gen))
    do, kv, dim, seqs = case["do"], case["kv"], case["dim"], case["seqs"]
    dtype = TYPES[case.get("type", "bf16")]
    normal = lambda *shape: torch.randn(shape, generator=gen, device=DEV, dtype=dtype)
    if do == "shared":
        s["k"], s["v"] = normal(s["pages"], s["page"], kv, dim), normal(s["pages"], s["page"], kv, dim)
        s["common"] = torch.tensor([_common(case)], device=DEV, dtype=torch.int32)
    else:
        s["k"], s["v"], s["scales"] = _packed(case, s["pages"], gen)
    if do == "evict":
        s["scores"] = _scores(case, s["pages"], gen)
        # (a cache that was evicted before: each head has its tokens in an order of its own)
        s["seen"] = s["lengths"] + 1000
        s["positions"] = _positions(s, gen)
        s["moves"], s["counts"] = _moves(s)
        return s
    if do == "read":
        s["starts"] = (s["lengths"] - case["tokens"]).clamp(min=0) if case["tail"] else torch.zeros_like(s["lengths"])
        s["out"] = [torch.zeros(seqs, case["tokens"], kv, dim, device=DEV, dtype=dtype) for _ in range(2)]
        return s
    new, heads = case["new"], case["heads"]
    s["count"] = torch.tensor(_counts(case), device=DEV, dtype=torch.int32) if case["ragged"] else None
    s["out"] = torch.zeros(seqs, new, heads, dim, device=DEV, dtype=dtype)
    if do in ("attend", "shared"):
        s["q"] = 2.0 * normal(seqs, new, heads, dim)
        s["scale"] = 1.0 / math.sqrt(dim)
        s["scores"] = _scores(case, s["pages"], gen) if case.get("book") else None
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
    s["starts"] = s["lengths"] - (s["count"] if case["ragged"] else new)
    s["back"] = [torch.zeros(seqs, new, kv, dim, device=DEV, dtype=dtype) for _ in range(2)]
    return s


def _handle(s):
    """The program's view of its cache, made once."""
    from paper_2310_09443_b200 import binding as g10
    if "handle" not in s:
        if s["do"] == "shared":
            s["handle"] = g10.CacheBuffers(s["k"], s["v"], s["table"], s["lengths"])
            s["ws"] = torch.empty(g10.g10_cache_shared_workspace_bytes(s["handle"], s["new"], s["heads"]), dtype=torch.uint8, device=DEV)
        else:
            s["handle"] = g10.PackedBuffers(s["k"], s["v"], s["scales"], s["table"], s["lengths"], dtype=TYPES[s.get("type", "bf16")], seen=s.get("seen"),
                                            scores=s.get("scores"), positions=s.get("positions"))
            if s["do"] == "attend":
                s["ws"] = torch.empty(g10.g10_packed_workspace_bytes(s["handle"], s["new"], s["heads"], window=s["window"], sinks=s["sinks"], add_scores=s["book"]),
                                      dtype=torch.uint8, device=DEV)
    return g10, s["handle"]


def run(s):
    do = s["do"]
    if not own:
        return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend, "evict": _plain_evict, "shared": _plain_shared}[do](s)
    g10, cache = _handle(s)
    if do == "write":
        g10.g10_packed_append(cache, s["new_k"], s["new_v"], s["new_q"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6, cos=s["cos"], sin=s["sin"],
                              interleaved=s["interleaved"], counts=s["count"], q_out=s["out"])
        g10.g10_packed_read(cache, s["new"], starts=s["starts"], k=s["back"][0], v=s["back"][1])
        return _written(s, s["out"], *s["back"])
    if do == "read":
        g10.g10_packed_read(cache, s["tokens"], starts=s["starts"], k=s["out"][0], v=s["out"][1])
        return dict(k=s["out"][0], v=s["out"][1])
    if do == "attend":
        g10.g10_packed_attend(cache, s["q"], scale=s["scale"], window=s["window"], sinks=s["sinks"], counts=s["count"], add_scores=s["book"],
                              out=s["out"], lse=s["lse"], ws=s["ws"])
        return _attended(s, s["out"], s["lse"])
    if do == "shared":
        g10.g10_cache_attend_shared(cache, s["q"], s["common"], scale=s["scale"], counts=s["count"], out=s["out"], lse=s["lse"], ws=s["ws"])
        return dict(out=s["out"], lse=s["lse"])
    g10.g10_packed_evict(cache, s["moves"], s["counts"])
    return _evicted(s)


def _attended(s, out, lse):
    return dict(out=out, lse=lse, scores=s["scores"]) if s["book"] else dict(out=out, lse=lse)


def _written(s, q, k, v):
    return dict(q=q, k=k, v=v, scales=s["scales"], scores=s["scores"], positions=s["positions"])


def _bytes(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _evicted(s):
    """(Codes are moved, not computed: whole numbers.)"""
    return dict(k=_bytes(s["k"]), v=_bytes(s["v"]), scales=s["scales"], scores=s["scores"], positions=s["positions"])


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _places(s):
    """Page and place in the page of every slot up to the longest sequence, and whether the sequence has the slot: [seqs, slots]."""
    at = torch.arange(s["longest"], device=DEV)
    return s["table"].long()[:, at // s["page"]].clamp(min=0), (at % s["page"]).expand(s["table"].shape[0], -1), at[None] < s["lengths"][:, None]


def _rows(s, side, page, place, there):
    """Rows [seqs, slots, kv, dim] of keys (0) or values (1) in 32 bits, zero where there is no token."""
    codes = s["kv"[side]]
    if "scales" not in s:
        return torch.where(there[:, :, None, None], codes[page, place].float(), 0.0)
    head = torch.arange(codes.shape[2], device=DEV)[None, None]
    x = _bytes(codes)[page, place].view(codes.dtype).float() * s["scales"][page[:, :, None], head, place[:, :, None], side][..., None]
    return torch.where(there[:, :, None, None], x, 0.0)


def _sees(s, slots):
    """Which of the slots each new token sees: [seqs, new, slots]."""
    new = s["q"].shape[1]
    count = s["count"] if s["count"] is not None else torch.full_like(s["lengths"], new)
    token = torch.arange(new, device=DEV)
    slot = (s["lengths"] - count)[:, None] + token[None]
    sees = (slots <= slot[:, :, None]) & (token[None] < count[:, None])[:, :, None] & (slots < s["lengths"][:, None, None])
    if s.get("window"):
        sees = sees & ((slots < s["sinks"]) | (slots > slot[:, :, None] - s["window"]))
    return sees


def _weights(score):
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = weight.sum(-1, keepdim=True)
    return weight / torch.where(total == 0.0, 1.0, total), (top + torch.log(total)).squeeze(-1)


def _plain_attend(s):
    page, place, there = _places(s)
    seqs, new, heads, dim = s["q"].shape
    kv = s["k"].shape[2]
    k, v = _rows(s, 0, page, place, there), _rows(s, 1, page, place, there)
    q = s["q"].float().view(seqs, new, kv, heads // kv, dim)
    score = torch.einsum("bnkgd,bckd->bkgnc", q, k) * s["scale"]
    weight, lse = _weights(torch.where(_sees(s, torch.arange(s["longest"], device=DEV))[:, None, None], score, -math.inf))
    out = torch.einsum("bkgnc,bckd->bnkgd", weight, v).reshape(seqs, new, heads, dim).to(s["q"].dtype)
    if s["book"]:
        head = torch.arange(kv, device=DEV)
        s["scores"].index_put_((page[:, :, None], head[None, None], place[:, :, None]), weight.sum((2, 3)).transpose(1, 2), accumulate=True)
    return _attended(s, out, lse.permute(0, 3, 1, 2).reshape(seqs, new, heads))


def _plain_shared(s):
    """One product over the shared rows for all sequences, one over each sequence's own; the weights are those of both together."""
    seqs, new, heads, dim = s["q"].shape
    kv, common = s["k"].shape[2], s["prefix"] // s["page"] * s["page"]
    page, place, there = _places(s)
    q = s["q"].float().view(seqs, new, kv, heads // kv, dim)
    k0, v0 = (_rows(s, side, page[:1, :common], place[:1, :common], there[:1, :common])[0] for side in (0, 1))
    k1, v1 = (_rows(s, side, page[:, common:], place[:, common:], there[:, common:]) for side in (0, 1))
    score = torch.cat([torch.einsum("bnkgd,ckd->bkgnc", q, k0), torch.einsum("bnkgd,bckd->bkgnc", q, k1)], -1) * s["scale"]
    weight, lse = _weights(torch.where(_sees(s, torch.arange(s["longest"], device=DEV))[:, None, None], score, -math.inf))
    out = torch.einsum("bkgnc,ckd->bnkgd", weight[..., :common], v0) + torch.einsum("bkgnc,bckd->bnkgd", weight[..., common:], v1)
    return dict(out=out.reshape(seqs, new, heads, dim).to(s["q"].dtype), lse=lse.permute(0, 3, 1, 2).reshape(seqs, new, heads))


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


def _plain_write(s):
    seqs, new = s["new_q"].shape[:2]
    count = s["count"] if s["count"] is not None else torch.full_like(s["lengths"], new)
    token = torch.arange(new, device=DEV)[None]
    there = token < count[:, None]
    slot = torch.where(there, (s["lengths"] - count)[:, None] + token, 0)
    # a token that does not count writes what is there already to a page that nobody has
    page = torch.where(there, s["table"].long().gather(1, (slot // s["page"]).long()), s["spare"])
    place = (slot % s["page"]).long()
    cos, sin = (None, None) if s["cos"] is None else (s["cos"][slot], s["sin"][slot])
    wide = there[:, :, None, None]
    q = torch.where(wide, _plain_turn(s["new_q"], s["q_weight"], cos, sin, s["interleaved"]).to(s["new_q"].dtype), 0.0)
    k, k_scale = _quantised(_plain_turn(s["new_k"], s["k_weight"], cos, sin, s["interleaved"]), s["code"])
    v, v_scale = _quantised(s["new_v"].float(), s["code"])
    for pool, codes in ((s["k"], k), (s["v"], v)):
        _bytes(pool)[page, place] = torch.where(wide, _bytes(codes), _bytes(pool)[page, place])
    one = there[:, :, None]
    s["scales"][page, :, place] = torch.where(wide, torch.stack([k_scale, v_scale], -1), s["scales"][page, :, place])
    s["scores"][page, :, place] = torch.where(one, 0.0, s["scores"][page, :, place])
    s["positions"][page, :, place] = torch.where(one, slot[:, :, None].int(), s["positions"][page, :, place])
    back = [torch.where(wide, _rows(s, side, page, place, there), 0.0).to(q.dtype) for side in (0, 1)]
    return _written(s, q, *back)


def _plain_read(s):
    slot = s["starts"][:, None] + torch.arange(s["tokens"], device=DEV)[None]
    there = slot < s["lengths"][:, None]
    slot = torch.where(there, slot, 0)
    page, place = s["table"].long().gather(1, (slot // s["page"]).long()), (slot % s["page"]).long()
    k, v = (_rows(s, side, page, place, there).to(TYPES[s["type"]]) for side in (0, 1))
    return dict(k=k, v=v)


def _positions(s, gen):
    """Positions of the tokens that a cache evicted before holds: as many of the tokens seen as it has slots, in any order."""
    page, place, there = _places(s)
    kv = s["k"].shape[2]
    mixed = torch.rand(there.shape[0], kv, s["longest"], generator=gen, device=DEV) + (~there[:, None]).float()
    rank = mixed.argsort(-1).argsort(-1).int()                                # [seqs, kv, slots]: 0 .. length - 1 where there is a token
    position = torch.where(rank < 500, rank, rank + 1000)
    out = torch.full((s["pages"], kv, s["page"]), -1, dtype=torch.int32, device=DEV)
    cell = (page[:, :, None].expand(-1, -1, kv)[there], torch.arange(kv, device=DEV).expand(there.shape + (kv,))[there], place[:, :, None].expand(-1, -1, kv)[there])
    out[cell] = position.transpose(1, 2)[there]
    return out


def _moves(s):
    """What a plan of evictions says: `budget` slots stay, the first and the last tokens and those of the largest scores; those of them that
    stand behind the budget move into the gaps before it."""
    page, place, there = _places(s)
    kv, budget = s["k"].shape[2], s["budget"]
    cell = (page[:, :, None], torch.arange(kv, device=DEV)[None, None], place[:, :, None])
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
    return moves[:, :, :budget].contiguous(), mover.sum(-1).int()


def _plain_evict(s):
    budget = s["budget"]
    real = torch.arange(budget, device=DEV) < s["counts"][:, :, None]
    seq = torch.arange(s["table"].shape[0], device=DEV)[:, None, None]
    head = torch.arange(s["k"].shape[2], device=DEV)[None, :, None].expand_as(real)
    # (an entry that is no move repeats the sequence's first move, or copies the first slot onto itself where there is none)
    source, target = (torch.where(real, s["moves"][..., side], 0).long() for side in (0, 1))
    found = s["table"].long()
    pages = [found[seq, x // s["page"]] for x in (source, target)]
    places = [x % s["page"] for x in (source, target)]
    same = ~real & (s["counts"] > 0)[:, :, None]
    pages = [torch.where(same, p[:, :, :1], p) for p in pages]
    places = [torch.where(same, p[:, :, :1], p) for p in places]
    for pool in (_bytes(s["k"]), _bytes(s["v"])):
        pool[pages[1], places[1], head] = pool[pages[0], places[0], head]
    for table in (s["scores"], s["positions"], s["scales"]):
        table[pages[1], head, places[1]] = table[pages[0], head, places[0]]
    return _evicted(s)


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    do = case["do"]
    lengths, table, page = s["lengths"].tolist(), s["table"].tolist(), s["page"]
    pick = lambda b, n: (torch.tensor(table[b], device=DEV).repeat_interleave(page)[:n].long(), torch.arange(n, device=DEV) % page)
    if do == "evict":
        scales, scores = s["scales"].double(), s["scores"].double()
        moves, counts = s["moves"].cpu(), s["counts"].tolist()
        for b in range(case["seqs"]):
            pages, places = pick(b, lengths[b])
            for h in range(case["kv"]):
                source, target = moves[b, h, :counts[b][h]].long().to(DEV).T
                for x in (scales, scores):
                    x[pages[target], h, places[target]] = x[pages[source], h, places[source]]
        return dict(k=None, v=None, scales=scales, scores=scores, positions=None)

    def row(side, pages, places, heads):
        """Rows in 64 bits."""
        x = s["kv"[side]]
        if do == "shared":
            return x[pages, places, heads].double()
        return x.view(torch.uint8)[pages, places, heads].view(x.dtype).double() * s["scales"][pages, heads, places, side].double()[..., None]

    if do == "read":
        out = [torch.zeros(s["out"][0].shape, dtype=torch.float64, device=DEV) for _ in range(2)]
        for b, start in enumerate(s["starts"].tolist()):
            pages, places = (x[start:start + case["tokens"], None] for x in pick(b, lengths[b]))
            for side in (0, 1):
                out[side][b, :len(pages)] = row(side, pages, places, torch.arange(case["kv"], device=DEV)[None])
        return dict(k=out[0], v=out[1])
    counts = _counts(case)
    group = case["heads"] // case["kv"]
    if do == "write":
        scales, scores = s["scales"].double(), s["scores"].double()
        q, k, v = (torch.zeros(x.shape, dtype=torch.float64, device=DEV) for x in (s["out"], *s["back"]))
        half = case["rotary"] // 2
        first = torch.arange(half, device=DEV) * (2 if case["interleaved"] else 1)
        second = first + (1 if case["interleaved"] else half)
        top = LARGEST[case["code"]]

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

        def nearest(x):
            """The nearest value that a code stands for, x in units of the scale; ties to even."""
            if case["code"] == "int8":
                return x.round()
            unit = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
            return (x / unit).round() * unit

        for b, (length, count) in enumerate(zip(lengths, counts)):
            pages, places = (x[length - count:] for x in pick(b, length))
            slots = torch.arange(length - count, length, device=DEV)
            q[b, :count] = turned(s["new_q"][b, :count], s["q_weight"], slots)
            for side, to, x in ((0, k, turned(s["new_k"][b, :count], s["k_weight"], slots)), (1, v, s["new_v"][b, :count].double())):
                scale = x.abs().amax(-1) / top
                to[b, :count] = nearest(x / scale[..., None]) * scale[..., None]
                scales[pages, :, places, side] = scale
            scores[pages, :, places] = 0.0
        return dict(q=q, k=k, v=v, scales=scales, scores=scores, positions=None)
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    scores = s["scores"].double() if case.get("book") else None
    for b, (length, count) in enumerate(zip(lengths, counts)):
        pages, places = pick(b, length)
        slot = torch.arange(length, device=DEV)
        for h in range(case["kv"]):
            k, v = row(0, pages, places, h), row(1, pages, places, h)
            mine = slice(h * group, (h + 1) * group)
            for t in range(count):
                p = length - count + t
                sees = slot <= p
                if case.get("window"):
                    sees = sees & ((slot < case["sinks"]) | (slot > p - case["window"]))
                logit = (s["q"][b, t, mine].double() @ k.T * s["scale"]).masked_fill(~sees, -math.inf)
                lse[b, t, mine] = logit.logsumexp(-1)
                weight = (logit - lse[b, t, mine, None]).exp()
                out[b, t, mine] = weight @ v
                if scores is not None:
                    scores[pages, h, places] += weight.sum(0)
    return dict(out=out, lse=lse, scores=scores) if case.get("book") else dict(out=out, lse=lse)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def work(case):
    """Each packed row, its scale, and each row of a shared beginning read once (read, attend, shared), each new token read, its codes, scales and
    queries written once, and read back (write), each moved row read and written once (evict; the share of the kept tokens that stand behind the
    budget is that of all)."""
    do, kv, lengths, dim = case["do"], case["kv"], _lengths(case), case["dim"]
    if do == "attend":
        slots, rows = sum(_visible(case)), case["new"] * case["heads"]
        n = slots * kv * (2 * dim + 8) + case["seqs"] * rows * (dim * 4 + 4) + (8 * slots * kv if case["book"] else 0)
        return {"bytes": n, "flops": 4 * sum(v * c for v, c in zip(_visible(case), _counts(case))) * case["heads"] * dim}
    if do == "shared":
        common, rows = _common(case), case["seqs"] * case["new"] * case["heads"]
        slots = common + sum(n - common for n in lengths)
        return {"bytes": slots * kv * dim * 4 + rows * (dim * 4 + 4), "flops": 4 * sum(n * c for n, c in zip(lengths, _counts(case))) * case["heads"] * dim}
    if do == "write":
        tokens = sum(_counts(case))
        return {"bytes": tokens * (case["heads"] * dim * 4 + kv * (2 * dim * 2 + 2 * (dim + 4) + 2 * dim * 2 + 8) + 4 * case["rotary"]),
                "flops": tokens * (case["heads"] + 2 * kv) * dim * 7}
    if do == "read":
        tokens = sum(min(case["tokens"], n) for n in lengths)
        return {"bytes": tokens * kv * 2 * (dim + 4) + case["seqs"] * case["tokens"] * kv * 4 * dim, "flops": tokens * kv * 2 * dim}
    moves = sum(case["budget"] * (n - case["budget"]) // n for n in lengths if n > case["budget"]) * kv
    return {"bytes": moves * (dim * 4 + 40), "flops": 0}
