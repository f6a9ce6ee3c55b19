"""The serving operators that keep a session's cache small, as cases that can be timed and checked.

What a scene's kept tokens left in the paged cache grows with every question and answer.  It is held in 4 bits, and the
tokens that no answer attends to are dropped.  Kinds of case:
  append4  cp.kv_append4: position rotation of queries and keys, keys and values into a 4-bit cache; what it holds then is read back
  gather   cp.kv_gather: keys and values of some slots of a paged cache as dense rows
  attend4  cp.paged_attention4: one new token of each sequence over its 4-bit keys and values
  mass     cp.paged_attention_mass: attention that also adds to each cached token the weight that it got
  evict    cp.kv_evict: the tokens of least accumulated weight leave the cache, the others close the gaps

A 4-bit cache holds e2m1 values (0, .5, 1, 1.5, 2, 3, 4, 6 and a sign; two a byte, the even dim in the low half) and, for each
32 dims of a token's head, the power of two that they are times of, as a byte (its exponent plus 127).

With `own` false the operators are computed in plain torch operations, in 32 bits; angles, rotated keys and what is compared
with the borders between two 4-bit values in 64.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "e2m1": torch.uint8}
E4M3_MAX = 448.0
# The exponents that a block of 32 may have: its values stay normal and finite in the type that it was made from.
EXPONENTS = {"bf16": (-125, 125), "f16": (-23, 13)}


def listed():
    return [
        # One decoded token of two requests, 28 heads of 128 on 4: a launch and little else.
        dict(name="append4_2", kind="append4", tokens=2, hq=28, hk=4, d=128, rot=128, page=16, span=6272, dtype="bf16",
             interleaved=False, magnitude=1.0, stretch=1.0),
        # A whole unpruned 6271-token prompt, every head with its own keys, half of each head rotated.
        dict(name="append4_6271_part", kind="append4", tokens=6271, hq=32, hk=32, d=64, rot=32, page=50, span=6271,
             dtype="f16", interleaved=True, magnitude=1.2, stretch=4.0),
        # The kept tokens (10 %) of a 16384-token scene, read back from 4 bits to go elsewhere.
        dict(name="gather_1638_e2m1", kind="gather", tokens=1638, hk=4, d=128, page=64, dtype="bf16", cache="e2m1"),
        # A long session of many scenes from 8 bits with odd pages.
        dict(name="gather_65537_e4m3", kind="gather", tokens=65537, hk=8, d=128, page=50, dtype="f16", cache="e4m3"),
        # One request that was pruned from 6272 tokens to 628, its first decoded token.
        dict(name="attend4_1x629", kind="attend4", batch=1, longest=629, shortest=629, hq=28, hk=4, d=128, page=16,
             dtype="bf16", window=0, lse=False),
        # Requests of very different lengths served together, every head with its own keys, odd pages.
        dict(name="attend4_24x6900_ragged", kind="attend4", batch=24, longest=6900, shortest=1, hq=16, hk=16, d=64, page=50,
             dtype="f16", window=0, lse=True),
        # A batch of long sessions: 544 MiB of codes and scales.
        dict(name="attend4_16x65536", kind="attend4", batch=16, longest=65536, shortest=60000, hq=28, hk=4, d=128, page=64,
             dtype="bf16", window=0, lse=False),
        # Three requests after a prune, 16 bits.
        dict(name="mass_3x1701", kind="mass", batch=3, longest=1701, shortest=629, hq=28, hk=4, d=128, page=16, dtype="bf16",
             cache="bf16", window=0),
        # One long session over many scenes, 4 bits.
        dict(name="mass_1x131072_e2m1", kind="mass", batch=1, longest=131072, shortest=131072, hq=28, hk=4, d=128, page=64,
             dtype="bf16", cache="e2m1", window=0),
        # A served batch drops 64 tokens each after as many decoded ones: the budget of a pruned scene again.
        dict(name="evict_8x1702", kind="evict", batch=8, longest=1702, shortest=1638, hk=4, d=128, page=16, dtype="bf16",
             cache="bf16", keep=1638, recent=128, sink=4),
        # Prompts of whole scenes cut to a tenth, odd pages, 8 bits; some are short enough already.
        dict(name="evict_5x16384_e4m3", kind="evict", batch=5, longest=16384, shortest=1001, hk=8, d=64, page=50, dtype="f16",
             cache="e4m3", keep=1639, recent=32, sink=0),
        # One long session halved, 4 bits, what is left read back.
        dict(name="evict_1x131072_e2m1", kind="evict", batch=1, longest=131072, shortest=131072, hk=4, d=128, page=64,
             dtype="bf16", cache="e2m1", keep=65536, recent=1024, sink=16),
    ]


def _log_size(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append4", "gather", "attend4", "attend4", "mass", "evict"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    d = rng.choice([64, 96, 128, 128, 192, 256])
    hk = rng.choice([1, 2, 4, 8, 16])
    hq = hk * rng.choice([1, 2, 3, 4, 7, 8] + ([16, 20] if hk <= 2 else []))
    page = rng.choice([1, 7, 16, 16, 32, 50, 64, 100, 128])
    cache = rng.choice([dtype, "e4m3", "e2m1"])
    if kind == "append4":
        tokens = _log_size(rng, 1, 6271 * 32 * 64 * 3 // ((hq + 2 * hk) * d))
        return dict(kind=kind, tokens=tokens, hq=hq, hk=hk, d=d, rot=rng.choice([d, d, d // 2, d // 4]), page=page,
                    span=tokens * rng.choice([1, 10, 100]) + rng.randint(0, 2000), dtype=dtype,
                    interleaved=rng.random() < 0.4, magnitude=rng.choice([1.0, 1.2]), stretch=rng.choice([1.0, 4.0, 8.0]))
    if kind == "gather":
        return dict(kind=kind, tokens=_log_size(rng, 1, 65537 * 8 * 128 // (hk * d)), hk=hk, d=d, page=page, dtype=dtype, cache=cache)
    batch = _log_size(rng, 1, 48)
    # Up to a quarter of the largest listed case.
    longest = _log_size(rng, 1, min(131072, 65536 * 4 * 128 * 4 // (batch * hk * d)))
    shortest = rng.choice([0, 1, longest // 2, longest])
    if kind == "evict":
        keep = max(1, min(_log_size(rng, 1, longest), longest * rng.choice([1, 3, 15]) // 16))
        recent = rng.choice([0, min(keep, 32), keep // 2])
        return dict(kind=kind, batch=batch, longest=longest, shortest=shortest, hk=hk, d=d, page=page, dtype=dtype, cache=cache,
                    keep=keep, recent=recent, sink=min(rng.choice([0, 4]), keep - recent))
    window = rng.choice([0, 0, 0, longest // 3 | 1])
    case = dict(kind=kind, batch=batch, longest=longest, shortest=shortest, hq=hq, hk=hk, d=d, page=page, dtype=dtype, window=window)
    return dict(case, lse=rng.random() < 0.5) if kind == "attend4" else dict(case, cache=cache)


# ---------------------------------------------------------------------------
# Inputs.

def _to8(x):
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _cut4(x, dtype):
    """Rows x [..., d] as 4-bit codes (one a byte) and exponents [..., d / 32]: per 32 dims the smallest power of two that
    six times reaches the largest, within the type's range; codes to nearest, ties to the even one."""
    low, high = EXPONENTS[dtype]
    block = x.unflatten(-1, (-1, 32))
    top, power = torch.frexp(block.abs().amax(-1))
    power = torch.where(top > 0, torch.where(top <= 0.75, power - 3, power - 2), low).clamp(low, high)
    y = torch.ldexp(block, -power[..., None])
    size = y.abs()
    code = torch.where(size < 2, torch.round(2 * size), torch.where(size < 4, torch.round(size) + 2, torch.round(size / 2) + 4))
    code = code.clamp(max=7).to(torch.uint8) + 8 * (y < 0).to(torch.uint8)
    return code.flatten(-2), power


def _pack4(code):
    return code[..., 0::2] | code[..., 1::2] << 4


def _value4(code, power):
    """What codes (one a byte) and exponents stand for, in 32 bits."""
    level = (code & 7).float()
    size = torch.where(level < 4, level / 2, torch.where(level < 6, level - 2, 2 * level - 8))
    value = torch.where(code >= 8, -size, size).unflatten(-1, (-1, 32))
    return (value * torch.exp2(power.float())[..., None]).flatten(-2)


def _open4(packed, scale):
    """The same from a cache's rows."""
    return _value4(torch.stack([packed & 15, packed >> 4], -1).flatten(-2), scale.int() - 127)


def _lengths(case):
    """The batch's lengths, evenly spread; which sequence has which is the seed's."""
    b = case["batch"]
    lo, hi = case["shortest"], case["longest"]
    return [hi - (hi - lo) * i // max(b - 1, 1) for i in range(b)]


def _make_cache(s, pages, normal, uniform):
    """Keys and values of recycled pages (slots past a sequence's end hold what was there before), and their scales."""
    hk, d, page, cache = s["hk"], s["d"], s["page"], s["cache"]
    s["k_scale"] = s["v_scale"] = None
    for name in ("k", "v"):
        if cache == "e4m3":
            s[name + "_scale"] = 0.01 + 0.02 * uniform(hk)
            s[name + "_cache"] = _to8(normal(pages, hk, page, d) / 0.02)
        elif cache == "e2m1":
            # A few dims of a head are louder than the others.
            loud = torch.where(uniform(hk, 1, d) < 0.03, 4.0, 1.0)
            codes = torch.empty(pages, hk, page, d // 2, dtype=torch.uint8, device=DEVICE)
            scales = torch.empty(pages, hk, page, d // 32, dtype=torch.uint8, device=DEVICE)
            step = max(1, (1 << 26) // (hk * page * d))
            for at in range(0, pages, step):
                code, power = _cut4(normal(min(step, pages - at), hk, page, d) * loud, s["dtype"])
                codes[at:at + step] = _pack4(code)
                scales[at:at + step] = (power + 127).to(torch.uint8)
            s[name + "_cache"], s[name + "_scale"] = codes, scales
        else:
            s[name + "_cache"] = normal(pages, hk, page, d).to(TYPES[cache])


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, generator=g)

    def uniform(*shape):
        return torch.rand(*shape, device=DEVICE, generator=g)

    kind, s = case["kind"], dict(case)
    t, hk, d, page = TYPES[case["dtype"]], case["hk"], case["d"], case["page"]
    s.setdefault("cache", "e2m1")
    if kind in ("append4", "gather"):
        tokens = case["tokens"]
        pages = (tokens + page - 1) // page + 2
        order = torch.randperm(pages, device=DEVICE, generator=g)
        at = torch.arange(tokens, device=DEVICE)
        s["slots"] = order[at // page] * page + at % page
        _make_cache(s, pages, normal, uniform)
        if kind == "gather":
            return s
        hq = case["hq"]
        # One projection's output, of which queries, keys and values are views.
        qkv = normal(tokens, (hq + 2 * hk) * d).to(t)
        s["q"] = qkv[:, :hq * d].view(tokens, hq, d)
        s["k"] = qkv[:, hq * d:(hq + hk) * d].view(tokens, hk, d)
        s["v"] = qkv[:, (hq + hk) * d:].view(tokens, hk, d)
        # Kept tokens: ascending positions with gaps.
        step = uniform(tokens).cumsum(0)
        s["positions"] = (step * ((case["span"] - 1) / step[-1])).to(torch.int32)
        s["inv_freq"] = 10000.0 ** (-torch.arange(0, case["rot"], 2, device=DEVICE) / case["rot"]) / case["stretch"]
        return s
    b = case["batch"]
    lengths = _lengths(case)
    order = torch.randperm(b, device=DEVICE, generator=g)
    width = max(1, (max(lengths) + page - 1) // page)
    pages = b * width + 1
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEVICE)[order]
    s["max_length"] = max(lengths)
    s["table"] = torch.randperm(pages, device=DEVICE, generator=g)[:b * width].view(b, width).to(torch.int32)
    _make_cache(s, pages, normal, uniform)
    if kind != "evict":
        s["q"] = normal(b, case["hq"], d).to(t)
    if kind == "mass":
        s["mass"] = uniform(b, hk, s["max_length"])
    if kind == "evict":
        span = s["max_length"]
        # Weight gathers on few tokens; those of the last step have none yet.
        mass = torch.exp(2.0 * normal(b, hk, span)) / span
        where = torch.arange(span, device=DEVICE)
        s["mass"] = torch.where(where < s["lengths"][:, None, None] - 1, mass, 0.0)
        s["mass_out"] = torch.empty_like(s["mass"])
        # Slots of the tokens that are left, for those who read them back.
        kept = (where < s["lengths"][:, None].clamp(max=case["keep"])).nonzero()
        s["kept_slots"] = s["table"][kept[:, 0], kept[:, 1] // page].long() * page + kept[:, 1] % page
    return s


# ---------------------------------------------------------------------------
# One pass.

def run(s):
    return (_run_own if own else _run_plain)[s["kind"]](s)


def _own_gather(s):
    import paper_2608_13226_amd as cp
    return list(cp.kv_gather(s["k_cache"], s["v_cache"], s["slots"], dtype=TYPES[s["dtype"]], k_scale=s["k_scale"], v_scale=s["v_scale"]))


def _rows_of(s, slots):
    """Keys and values [slots, heads, d] in 32 bits."""
    page, at = slots // s["page"], slots % s["page"]
    rows = []
    for cache, scale in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"])):
        if s["cache"] == "e2m1":
            rows.append(_open4(cache[page, :, at], scale[page, :, at]))
        elif s["cache"] == "e4m3":
            rows.append(cache.view(torch.uint8)[page, :, at].view(torch.float8_e4m3fn).float() * scale[:, None])
        else:
            rows.append(cache[page, :, at].float())
    return rows


def _plain_gather(s):
    return [x.to(TYPES[s["dtype"]]) for x in _rows_of(s, s["slots"])]


def _own_append4(s):
    import paper_2608_13226_amd as cp
    q = cp.kv_append4(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["inv_freq"], s["k_cache"], s["v_cache"], s["k_scale"],
                      s["v_scale"], interleaved=s["interleaved"], magnitude=s["magnitude"])
    return [q, *_own_gather(s)]


def _turn(x, cos, sin, s):
    part, rest = x[..., :s["rot"]], x[..., s["rot"]:]
    if s["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = part[..., :s["rot"] // 2], part[..., s["rot"] // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, rest], -1)


def _plain_append4(s):
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = s["magnitude"] * angle.cos()[:, None], s["magnitude"] * angle.sin()[:, None]
    q = _turn(s["q"].float(), cos.float(), sin.float(), s).to(s["q"].dtype)
    page, at = s["slots"] // s["page"], s["slots"] % s["page"]
    values = []
    for x, cache, scale in ((_turn(s["k"].double(), cos, sin, s), s["k_cache"], s["k_scale"]), (s["v"].float(), s["v_cache"], s["v_scale"])):
        code, power = _cut4(x, s["dtype"])
        cache[page, :, at] = _pack4(code)
        scale[page, :, at] = (power + 127).to(torch.uint8)
        values.append(_value4(code, power).to(s["q"].dtype))
    return [q, *values]


def _own_attend4(s):
    import paper_2608_13226_amd as cp
    return cp.paged_attention4(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["lengths"],
                               max_length=s["max_length"], window=s["window"], return_lse=s["lse"])


def _cached(s, cache, scale):
    """What a sequence's pages hold, [batch, heads, span, d] in 32 bits."""
    at = s["table"].long()
    if s["cache"] == "e4m3":
        x = cache.view(torch.uint8)[at].view(torch.float8_e4m3fn).float() * scale[:, None, None]
    else:
        x = _open4(cache[at], scale[at]) if s["cache"] == "e2m1" else cache[at].float()
    return x.transpose(1, 2).flatten(2, 3)


def _weights(s):
    """Which tokens count, the softmax's weights [batch, heads, group, span] and log of its sums."""
    b, hk = s["batch"], s["hk"]
    k = _cached(s, s["k_cache"], s["k_scale"])
    score = torch.matmul(s["q"].float().view(b, hk, -1, s["d"]), k.transpose(2, 3)) / math.sqrt(s["d"])
    where = torch.arange(k.shape[2], device=DEVICE)
    seen = where < s["lengths"][:, None]
    if s["window"]:
        seen = seen & (where >= s["lengths"][:, None] - s["window"])
    seen = seen[:, None, None, :]
    score = torch.where(seen, score, -math.inf)
    top = score.amax(3, keepdim=True)
    p = torch.where(seen, torch.exp(score - top), 0.0)
    total = p.sum(3, keepdim=True)
    return seen, p / torch.where(total > 0, total, 1.0), (top + total.log()).flatten(1)


def _plain_attend(s):
    seen, p, lse = _weights(s)
    v = torch.where(seen.transpose(2, 3), _cached(s, s["v_cache"], s["v_scale"]), 0.0)
    o = torch.matmul(p, v).view(s["batch"], s["hq"], s["d"]).to(s["q"].dtype)
    return p, o, lse


def _plain_attend4(s):
    _, o, lse = _plain_attend(s)
    return [o, lse] if s["lse"] else o


def _own_mass(s):
    import paper_2608_13226_amd as cp
    o = cp.paged_attention_mass(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["mass"], max_length=s["max_length"],
                                window=s["window"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return [o, s["mass"]]


def _plain_mass(s):
    p, o, _ = _plain_attend(s)
    s["mass"] += p.sum(2)[:, :, :s["max_length"]]
    return [o, s["mass"]]


def _own_evict(s):
    import paper_2608_13226_amd as cp
    r = cp.kv_evict(s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["mass"], s["keep"], recent=s["recent"], sink=s["sink"],
                    max_length=s["max_length"], k_scale=s["k_scale"] if s["cache"] == "e2m1" else None,
                    v_scale=s["v_scale"] if s["cache"] == "e2m1" else None, mass_out=s["mass_out"])
    return [r.kept, r.lengths, r.mass, *_left(s, cp.kv_gather if s["cache"] == "e2m1" else None)]


def _left(s, gather):
    """The caches; of 4-bit ones the values that are left."""
    if s["cache"] != "e2m1":
        return [s["k_cache"], s["v_cache"]]
    if gather:
        return list(gather(s["k_cache"], s["v_cache"], s["kept_slots"], dtype=TYPES[s["dtype"]], k_scale=s["k_scale"], v_scale=s["v_scale"]))
    return [x.to(TYPES[s["dtype"]]) for x in _rows_of(s, s["kept_slots"])]


def _plain_evict(s):
    b, hk, keep, page = s["batch"], s["hk"], s["keep"], s["page"]
    span = s["mass"].shape[2]
    n = s["lengths"].long()[:, None, None]
    left = n.clamp(max=keep)
    at = torch.arange(span, device=DEVICE).expand(b, hk, span)
    valid, late = at < n, at >= n - s["recent"]
    # Tokens that stay before any weight, NaN after all of them, what is no token last; equal ones by their place.
    rank = torch.where(torch.isnan(s["mass"]), -1.5e300, s["mass"].double().clamp(-1e300, 1e300))
    rank = torch.where(valid, torch.where(late | (at < s["sink"]), 2e300, rank), -2e300)
    order = torch.sort(rank, dim=2, descending=True, stable=True).indices
    stays = torch.zeros(b, hk, span, dtype=torch.bool, device=DEVICE).scatter(2, order, at < left)
    # Where tokens stay in place, which places fall vacant before the last `recent`, and who moves there.
    front = torch.where(n > keep, keep - s["recent"], n)
    hole = ~stays & (at < front)
    mover = stays & (at >= front) & ~late
    mover_rank = torch.where(mover, mover.cumsum(2) - 1, span)
    movers = torch.zeros(b, hk, span + 1, dtype=torch.long, device=DEVICE).scatter(2, mover_rank, at)
    hole_rank = torch.where(hole, hole.cumsum(2) - 1, span)
    source = torch.where(hole, movers.gather(2, hole_rank), at)
    source = torch.where((at >= front) & (at < left), n - s["recent"] + at - front, source)
    there = at < left
    kept = torch.full((b, hk, keep), -1, dtype=torch.int32, device=DEVICE)
    kept[:, :, :span] = torch.where(there, source, -1)[:, :, :keep]
    source = torch.where(there, source, at)
    mass = torch.where(there, s["mass"].gather(2, source), 0.0)
    s["mass_out"].copy_(mass)
    to_page = s["table"].long()[:, None].expand(b, hk, -1).gather(2, at // page)
    from_page = s["table"].long()[:, None].expand(b, hk, -1).gather(2, source // page)
    head = torch.arange(hk, device=DEVICE)[None, :, None].expand(b, hk, span)
    scales = [s["k_scale"], s["v_scale"]] if s["cache"] == "e2m1" else []
    for cache in [s["k_cache"], s["v_cache"], *scales]:
        raw = cache.view(torch.uint8) if s["cache"] == "e4m3" else cache
        raw[to_page[there], head[there], at[there] % page] = raw[from_page[there], head[there], source[there] % page]
    return [kept, left.view(b).to(torch.int32), s["mass_out"], *_left(s, None)]


_run_own = {"append4": _own_append4, "gather": _own_gather, "attend4": _own_attend4, "mass": _own_mass, "evict": _own_evict}
_run_plain = {"append4": _plain_append4, "gather": _plain_gather, "attend4": _plain_attend4, "mass": _plain_mass, "evict": _plain_evict}


# ---------------------------------------------------------------------------
# What a pass cannot do without.

def _row_bytes(d, cache):
    return {"e2m1": d // 2 + d // 32, "e4m3": d}.get(cache, 2 * d)


def work(case):
    kind, hk, d = case["kind"], case["hk"], case["d"]
    row = _row_bytes(d, case.get("cache", "e2m1"))
    if kind == "append4":
        t, hq = case["tokens"], case["hq"]
        # What was written is read again and handed out.
        return {"bytes": t * ((2 * hq + 2 * hk) * d * 2 + 2 * hk * row + 12) + t * (2 * hk * (row + 2 * d) + 8) + 2 * case["rot"],
                "flops": 3 * t * (hq + hk) * case["rot"] + 4 * t * hk * d}
    if kind == "gather":
        return {"bytes": case["tokens"] * (2 * hk * (row + 2 * d) + 8), "flops": 2 * case["tokens"] * hk * d}
    b, lengths = case["batch"], _lengths(case)
    if kind == "evict":
        keep, recent, span = case["keep"], case["recent"], max(lengths)
        moved = 0.0
        for n in lengths:
            if n > keep:
                # Of the places before the last `recent` that many fall vacant, where weight does not go by place.
                free = max(1, n - recent - case["sink"])
                moved += recent + max(0, keep - recent - case["sink"]) * (n - keep) / free
        out = 2 * hk * sum(min(n, keep) for n in lengths) * (row + 2 * d) if case["cache"] == "e2m1" else 0
        return {"bytes": 4 * hk * (sum(lengths) + b * span + b * keep) + 8 * b + 4 * hk * moved * row + out, "flops": hk * sum(lengths)}
    hq = case["hq"]
    seen = [min(n, case["window"] or n) for n in lengths]
    pages = sum((n + case["page"] - 1) // case["page"] for n in seen)
    scales = 8 * hk if case.get("cache") == "e4m3" else 0
    more = 8 * hk * sum(seen) if kind == "mass" else 4 * b * hq if case["lse"] else 0
    return {"bytes": 2 * sum(seen) * hk * row + 4 * b * hq * d + 4 * pages + 4 * b + scales + more, "flops": 4 * sum(seen) * hq * d}


# ---------------------------------------------------------------------------
# The definitions in 64 bits.

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact4(cache, scale):
    """Rows of a 4-bit cache: each code's level, its sign, and the block's power of two."""
    levels = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64, device=DEVICE)
    x = torch.empty(*cache.shape[:-1], 2 * cache.shape[-1], dtype=torch.float64, device=DEVICE)
    x[..., 0::2] = levels[(cache % 16).long()]
    x[..., 1::2] = levels[(cache // 16).long()]
    return x * torch.pow(2.0, scale.double() - 127).repeat_interleave(32, -1)


def _exact_rows(s, name, page, head, off):
    cache, scale = s[name + "_cache"], s[name + "_scale"]
    if s["cache"] == "e2m1":
        return _exact4(cache[page, head, off], scale[page, head, off])
    if s["cache"] == "e4m3":
        return cache.view(torch.uint8)[page, head, off].view(torch.float8_e4m3fn).double() * scale[head].double()
    return cache[page, head, off].double()


def exact(case, seed):
    s = prepare(case, seed)
    return {"append4": _exact_append4, "gather": _exact_gather, "attend4": _exact_attend4, "mass": _exact_mass,
            "evict": _exact_evict}[case["kind"]](s)


def _exact_gather(s):
    page, off = s["slots"] // s["page"], s["slots"] % s["page"]
    return [torch.stack([_exact_rows(s, name, page, h, off) for h in range(s["hk"])], 1) for name in ("k", "v")]


def _exact_code(x, dtype):
    """The 4-bit value nearest to each x, in blocks of 32; of two as near the one with the even code."""
    low, high = EXPONENTS[dtype]
    unit = torch.full((*x.shape[:-1], x.shape[-1] // 32), 2.0 ** low, dtype=torch.float64, device=DEVICE)
    top = x.abs().unflatten(-1, (-1, 32)).amax(-1)
    for e in range(low, high):
        unit = torch.where(top > 6 * unit, 2 * unit, unit)
        if not bool((top > 6 * unit).any()):
            break
    unit = unit.repeat_interleave(32, -1)
    y = x.abs() / unit
    code = torch.zeros_like(y)
    for i in range(7):
        middle = (LEVELS[i] + LEVELS[i + 1]) / 2
        code += (y >= middle if i % 2 else y > middle).double()
    return torch.sign(x) * torch.tensor(LEVELS, dtype=torch.float64, device=DEVICE)[code.long()] * unit


def _exact_append4(s):
    half = s["rot"] // 2
    i = torch.arange(half, device=DEVICE)
    first, second = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + half)
    angle = torch.outer(s["positions"].double(), s["inv_freq"].double())
    turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle)[:, None]

    def turned(x):
        x = x.double().clone()
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    return [turned(s["q"]), _exact_code(turned(s["k"]), s["dtype"]), _exact_code(s["v"].double(), s["dtype"])]


def _exact_attend(s):
    group, page = s["hq"] // s["hk"], s["page"]
    out = torch.zeros(s["batch"], s["hq"], s["d"], dtype=torch.float64, device=DEVICE)
    lse = torch.full((s["batch"], s["hq"]), -math.inf, dtype=torch.float64, device=DEVICE)
    mass = s["mass"].double() if s["kind"] == "mass" else None
    for b, n in enumerate(s["lengths"].tolist()):
        low = max(0, n - s["window"]) if s["window"] else 0
        if n <= low:
            continue
        at = torch.arange(low, n, device=DEVICE)
        pg, off = s["table"][b].long()[at // page], at % page
        for h in range(s["hk"]):
            k, v = _exact_rows(s, "k", pg, h, off), _exact_rows(s, "v", pg, h, off)
            rows = slice(h * group, (h + 1) * group)
            score = (k @ s["q"][b, rows].double().t().contiguous()).t() / math.sqrt(s["d"])
            p = torch.softmax(score, 1)
            lse[b, rows] = torch.logsumexp(score, 1)
            out[b, rows] = p @ v
            if mass is not None:
                mass[b, h, low:n] += p.sum(0)
    return out, lse, mass


def _exact_attend4(s):
    out, lse, _ = _exact_attend(s)
    return [out, lse] if s["lse"] else out


def _exact_mass(s):
    out, _, mass = _exact_attend(s)
    return [out, mass]


def _exact_evict(s):
    keep, recent, page = s["keep"], s["recent"], s["page"]
    kept = torch.full((s["batch"], s["hk"], keep), -1, dtype=torch.int32)
    mass = torch.zeros(s["mass"].shape, dtype=torch.float64)
    for b, n in enumerate(s["lengths"].tolist()):
        for h in range(s["hk"]):
            w = s["mass"][b, h, :n].tolist()
            places = list(range(n))
            if n > keep:
                safe = set(range(s["sink"])) | set(range(n - recent, n))
                others = [j for j in range(n) if j not in safe]
                others.sort(key=lambda j: (-w[j], j))
                chosen = safe | set(others[:keep - len(safe)])
                movers = iter([j for j in range(keep - recent, n - recent) if j in chosen])
                places = [j if j in chosen else next(movers) for j in range(keep - recent)] + list(range(n - recent, n))
            kept[b, h, :len(places)] = torch.tensor(places, dtype=torch.int32)
            mass[b, h, :len(places)] = torch.tensor([w[j] for j in places], dtype=torch.float64)
    kept, mass = kept.to(DEVICE), mass.to(DEVICE)
    lengths = s["lengths"].clamp(max=keep)
    found = []
    for name in ("k", "v"):
        cache = s[name + "_cache"]
        new = cache.view(torch.uint8).clone().view(cache.dtype) if s["cache"] != "e2m1" else None
        rows = []
        for b, m in enumerate(lengths.tolist()):
            j = torch.arange(m, device=DEVICE)
            per_head = []
            for h in range(s["hk"]):
                old = kept[b, h, :m].long()
                where = s["table"][b].long()[old // page], h, old % page
                if new is None:
                    per_head.append(_exact_rows(s, name, *where))
                else:
                    new.view(torch.uint8)[s["table"][b].long()[j // page], h, j % page] = cache.view(torch.uint8)[where]
            if new is None:
                rows.append(torch.stack(per_head, 1))
        found.append(torch.cat(rows) if new is None else new.double())
    return [kept, lengths, mass, *found]
