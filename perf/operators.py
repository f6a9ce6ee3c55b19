"""The serving operators that follow a prune, as cases that can be timed and checked.

A pruned scene's tokens are read by a language model: their keys and values are put into a paged cache at the
positions they had in the video, and answers are decoded token by token from it.  Kinds of case:
  norm    cp.rms_norm: root-mean-square norm with the residual's addition, in the input's type or in 8 bits with row scales
  matvec  cp.w4_matvec: a few rows times 4-bit weights with group scales
  append  cp.kv_append: position rotation of queries and keys, keys and values into the paged cache
  attend  cp.paged_attention: one new token of each sequence over its paged keys and values

With `own` false the operators are computed in plain torch operations, in 32 bits.  8-bit values are e4m3 throughout.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}
E4M3_MAX = 448.0


def listed():
    return [
        # One decoded token of one request: a launch and little else.
        dict(name="norm_1x3584", kind="norm", rows=1, d=3584, dtype="bf16", out="bf16", residual=True),
        # A prompt of 32 frames of 14 x 14 tokens at a language model's width, for 8-bit products.
        dict(name="norm_6272x3584_e4m3", kind="norm", rows=6272, d=3584, dtype="bf16", out="e4m3", residual=True),
        # Queries, keys and values of one decoded token: 28 heads of 128 and 2 x 4 of them from 3584.
        dict(name="matvec_1x3584x4608", kind="matvec", m=1, k=3584, n=4608, group=128, x="bf16", dtype="bf16",
             out="bf16", zero=False),
        # Five requests, sizes that no tile divides, small groups with zero points, 8-bit rows, 32-bit results.
        dict(name="matvec_5x1184x1500_e4m3", kind="matvec", m=5, k=1184, n=1500, group=32, x="e4m3", dtype="bf16",
             out="f32", zero=True),
        # A full batch through a wide hidden layer (2 x 4 times the width).
        dict(name="matvec_64x3584x28672_f16", kind="matvec", m=64, k=3584, n=28672, group=64, x="f16", dtype="f16",
             out="f16", zero=True),
        # One decoded token of three requests.
        dict(name="append_3", kind="append", tokens=3, hq=28, hk=4, d=128, rot=128, page=16, span=6272, dtype="bf16",
             cache="bf16", interleaved=False, magnitude=1.0, stretch=1.0),
        # The kept tokens of a 16384-token scene (10 %) at their own positions, 8-bit cache, stretched positions.
        dict(name="append_1638_e4m3", kind="append", tokens=1638, hq=28, hk=4, d=128, rot=128, page=64, span=16384,
             dtype="bf16", cache="e4m3", interleaved=False, magnitude=1.2, stretch=4.0),
        # A whole unpruned 6271-token prompt, every head with its own keys, half of each head rotated.
        dict(name="append_6271_part", kind="append", tokens=6271, hq=32, hk=32, d=64, rot=32, page=50, span=6271,
             dtype="f16", cache="f16", interleaved=True, magnitude=1.0, stretch=1.0),
        # One request that was pruned from 6272 tokens to 628, its first decoded token.
        dict(name="attend_1x629", kind="attend", batch=1, longest=629, shortest=629, hq=28, hk=4, d=128, page=16,
             dtype="bf16", cache="bf16", window=0, lse=False),
        # Requests of very different lengths served together, every head with its own keys, odd pages.
        dict(name="attend_24x6900_ragged", kind="attend", batch=24, longest=6900, shortest=1, hq=16, hk=16, d=64,
             page=50, dtype="f16", cache="f16", window=0, lse=True),
        # One long session over many scenes, 8-bit cache.
        dict(name="attend_1x131072_e4m3", kind="attend", batch=1, longest=131072, shortest=131072, hq=28, hk=4, d=128,
             page=64, dtype="bf16", cache="e4m3", window=0, lse=False),
        # A batch of long sessions: 2 GiB of keys and values.
        dict(name="attend_16x65536", kind="attend", batch=16, longest=65536, shortest=60000, hq=28, hk=4, d=128,
             page=64, dtype="bf16", cache="bf16", window=0, lse=False),
    ]


def _log_size(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def draw(rng):
    kind = rng.choice(["norm", "matvec", "append", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind == "norm":
        d = rng.choice([256, 512, 1000, 1152, 1536, 2048, 3584, 4096, 5120, 8192, 2 * rng.randint(50, 2000) + 1])
        return dict(kind=kind, rows=_log_size(rng, 1, min(6272, 6272 * 3584 // d)), d=d, dtype=rng.choice([dtype, dtype, "f32"]),
                    out=rng.choice(["e4m3", "same"]), residual=rng.random() < 0.7)
    if kind == "matvec":
        group = rng.choice([32, 64, 128, 128, 256])
        k = group * max(1, _log_size(rng, 256, 16384) // group)
        n = _log_size(rng, 64, min(28672, 28672 * 3584 // k))
        k, n = (k + group if k == 3072 else k), (n + 1 if n == 3072 else n)
        return dict(kind=kind, m=_log_size(rng, 1, 64), k=k, n=n, group=group, x=rng.choice([dtype, dtype, "e4m3"]),
                    dtype=dtype, out=rng.choice([dtype, dtype, "f32"]), zero=rng.random() < 0.5)
    d = rng.choice([64, 96, 128, 128, 192, 256])
    hk = rng.choice([1, 2, 4, 8, 16])
    hq = hk * rng.choice([1, 2, 3, 4, 7, 8] + ([16, 20] if hk <= 2 else []))
    d = next(w for w in (d, 128, 64, 192, 256) if 3072 not in (hq * w, hk * w, (hq + 2 * hk) * w))
    page = rng.choice([1, 7, 16, 16, 32, 50, 64, 100, 128])
    cache = rng.choice([dtype, dtype, "e4m3"])
    if kind == "append":
        tokens = _log_size(rng, 1, 6271 * 32 * 64 * 3 // ((hq + 2 * hk) * d))
        return dict(kind=kind, tokens=tokens, hq=hq, hk=hk, d=d, rot=rng.choice([d, d, d // 2, d // 4]), page=page,
                    span=tokens * rng.choice([1, 10, 100]) + rng.randint(0, 2000), dtype=dtype, cache=cache,
                    interleaved=rng.random() < 0.4, magnitude=rng.choice([1.0, 1.2]), stretch=rng.choice([1.0, 4.0, 8.0]))
    batch = _log_size(rng, 1, 48)
    # Up to a quarter of the largest listed case.
    longest = _log_size(rng, 1, min(131072, 65536 * 4 * 128 * 4 // (batch * hk * d)))
    window = rng.choice([0, 0, 0, longest // 3 | 1])
    return dict(kind=kind, batch=batch, longest=longest, shortest=rng.choice([0, 1, longest // 2, longest]), hq=hq, hk=hk, d=d,
                page=page, dtype=dtype, cache=cache, window=window, lse=rng.random() < 0.5)


# ---------------------------------------------------------------------------
# Inputs.

def _to8(x):
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _lengths(case):
    """The batch's lengths, evenly spread; which sequence has which is the seed's."""
    b = case["batch"]
    lo, hi = case["shortest"], case["longest"]
    return [hi - (hi - lo) * i // max(b - 1, 1) for i in range(b)]


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, generator=g)

    def uniform(*shape):
        return torch.rand(*shape, device=DEVICE, generator=g)

    kind, s = case["kind"], dict(case)
    if kind == "norm":
        t = TYPES[case["dtype"]]
        # A residual stream: a few channels are far larger than the others.
        loud = torch.where(uniform(case["d"]) < 0.005, 30.0, 1.0)
        s["x"] = normal(case["rows"], case["d"]).to(t)
        s["weight"] = (1.0 + 0.2 * normal(case["d"])).to(t)
        s["h"] = (4.0 * loud * normal(case["rows"], case["d"])).to(t) if case["residual"] else None
        s["eps"] = 1e-6
    elif kind == "matvec":
        m, k, n, group = case["m"], case["k"], case["n"], case["group"]
        t = TYPES[case["dtype"]]
        x = normal(m, k)
        if case["x"] == "e4m3":
            s["x_scale"] = x.abs().amax(1) / E4M3_MAX
            s["x"] = _to8(x / s["x_scale"][:, None])
        else:
            s["x_scale"], s["x"] = None, x.to(t)
        # Two codes a byte along k, the even one in the low half.
        s["weight"] = torch.randint(0, 256, (n, k // 2), device=DEVICE, generator=g, dtype=torch.uint8)
        s["scale"] = ((0.5 + uniform(n, k // group)) / (4.0 * math.sqrt(k))).to(t)
        s["zero"] = (torch.randint(4, 12, (n, k // group), device=DEVICE, generator=g, dtype=torch.uint8)
                     if case["zero"] else None)
    elif kind == "append":
        t, c = TYPES[case["dtype"]], TYPES[case["cache"]]
        tokens, hq, hk, d, page = case["tokens"], case["hq"], case["hk"], case["d"], case["page"]
        # One projection's output, of which queries, keys and values are views.
        qkv = normal(tokens, (hq + 2 * hk) * d).to(t)
        s["q"] = qkv[:, :hq * d].view(tokens, hq, d)
        s["k"] = qkv[:, hq * d:(hq + hk) * d].view(tokens, hk, d)
        s["v"] = qkv[:, (hq + hk) * d:].view(tokens, hk, d)
        # Kept tokens: ascending positions with gaps.
        step = uniform(tokens).cumsum(0)
        s["positions"] = (step * ((case["span"] - 1) / step[-1])).to(torch.int32)
        pages = (tokens + page - 1) // page + 2
        order = torch.randperm(pages, device=DEVICE, generator=g)
        at = torch.arange(tokens, device=DEVICE)
        s["slots"] = order[at // page] * page + at % page
        s["inv_freq"] = 10000.0 ** (-torch.arange(0, case["rot"], 2, device=DEVICE) / case["rot"]) / case["stretch"]
        s["k_cache"] = normal(pages, hk, page, d).to(c)
        s["v_cache"] = normal(pages, hk, page, d).to(c)
        eight = case["cache"] == "e4m3"
        s["k_scale"] = (0.01 + 0.02 * uniform(hk)) if eight else None
        s["v_scale"] = (0.01 + 0.02 * uniform(hk)) if eight else None
    else:
        t, c = TYPES[case["dtype"]], TYPES[case["cache"]]
        b, hq, hk, d, page = case["batch"], case["hq"], case["hk"], case["d"], case["page"]
        lengths = _lengths(case)
        width = max(1, (max(lengths) + page - 1) // page)
        pages = b * width + 1
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEVICE)[torch.randperm(b, device=DEVICE, generator=g)]
        s["max_length"] = max(lengths)
        s["table"] = torch.randperm(pages, device=DEVICE, generator=g)[:b * width].view(b, width).to(torch.int32)
        s["q"] = normal(b, hq, d).to(t)
        eight = case["cache"] == "e4m3"
        s["k_scale"] = (0.01 + 0.02 * uniform(hk)) if eight else None
        s["v_scale"] = (0.01 + 0.02 * uniform(hk)) if eight else None
        # Pages are recycled: slots past a sequence's end hold what was there before.
        if eight:
            s["k_cache"] = _to8(normal(pages, hk, page, d) / 0.02)
            s["v_cache"] = _to8(normal(pages, hk, page, d) / 0.02)
        else:
            s["k_cache"] = torch.empty(pages, hk, page, d, dtype=c, device=DEVICE).normal_(generator=g)
            s["v_cache"] = torch.empty(pages, hk, page, d, dtype=c, device=DEVICE).normal_(generator=g)
    return s


# ---------------------------------------------------------------------------
# One pass.

def run(s):
    return (_run_own if own else _run_plain)[s["kind"]](s)


def _out_type(s):
    return s["dtype"] if s["out"] == "same" else s["out"]


def _own_norm(s):
    import paper_2608_13226_amd as cp
    r = cp.rms_norm(s["x"], s["weight"], eps=s["eps"], residual=s["h"], quantize=s["out"] == "e4m3")
    return [r.out, r.scale, r.residual]


def _plain_norm(s):
    h = s["x"].float()
    if s["h"] is not None:
        h = h + s["h"].float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + s["eps"]) * s["weight"].float()
    kept = None if s["h"] is None else h.to(s["x"].dtype)
    if s["out"] != "e4m3":
        return [y.to(s["x"].dtype), None, kept]
    scale = y.abs().amax(1) / E4M3_MAX
    return [_to8(y / scale[:, None]), scale, kept]


def _own_matvec(s):
    import paper_2608_13226_amd as cp
    return cp.w4_matvec(s["x"], s["weight"], s["scale"], zero=s["zero"], x_scale=s["x_scale"], out_dtype=TYPES[s["out"]])


def _plain_matvec(s):
    n, k = s["n"], s["k"]
    codes = torch.stack([s["weight"] & 15, s["weight"] >> 4], 2).view(n, s["k"] // s["group"], s["group"]).float()
    zero = 8.0 if s["zero"] is None else s["zero"].float()[:, :, None]
    w = ((codes - zero) * s["scale"].float()[:, :, None]).view(n, k)
    y = torch.matmul(s["x"].float(), w.t())
    if s["x_scale"] is not None:
        y = y * s["x_scale"][:, None]
    return y.to(TYPES[s["out"]])


def _own_append(s):
    import paper_2608_13226_amd as cp
    q = cp.kv_append(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["inv_freq"], s["k_cache"], s["v_cache"],
                     interleaved=s["interleaved"], magnitude=s["magnitude"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return [q, s["k_cache"], s["v_cache"]]


def _turn(x, cos, sin, s):
    x = x.float()
    part, rest = x[..., :s["rot"]], x[..., s["rot"]:]
    if s["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = part[..., :s["rot"] // 2], part[..., s["rot"] // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, rest], -1)


def _plain_append(s):
    angle = s["positions"].float()[:, None] * s["inv_freq"]
    cos, sin = s["magnitude"] * angle.cos()[:, None], s["magnitude"] * angle.sin()[:, None]
    q = _turn(s["q"], cos, sin, s).to(s["q"].dtype)
    page, at = s["slots"] // s["page"], s["slots"] % s["page"]
    for x, cache, scale in ((_turn(s["k"], cos, sin, s), s["k_cache"], s["k_scale"]), (s["v"].float(), s["v_cache"], s["v_scale"])):
        if scale is None:
            cache[page, :, at] = x.to(cache.dtype)
        else:
            cache.view(torch.uint8)[page, :, at] = _to8(x / scale[:, None]).view(torch.uint8)
    return [q, s["k_cache"], s["v_cache"]]


def _own_attend(s):
    import paper_2608_13226_amd as cp
    return cp.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], max_length=s["max_length"],
                              window=s["window"], k_scale=s["k_scale"], v_scale=s["v_scale"], return_lse=s["lse"])


def _plain_attend(s):
    b, hq, hk, d = s["batch"], s["hq"], s["hk"], s["d"]
    at = s["table"].long()
    span = at.shape[1] * s["page"]
    k = s["k_cache"].view(s["k_cache"].shape[0], -1)[at] if s["cache"] != "e4m3" else s["k_cache"].view(torch.uint8)[at].view(torch.float8_e4m3fn)
    v = s["v_cache"].view(s["v_cache"].shape[0], -1)[at] if s["cache"] != "e4m3" else s["v_cache"].view(torch.uint8)[at].view(torch.float8_e4m3fn)
    k = k.view(b, -1, hk, s["page"], d).transpose(1, 2).float().reshape(b, hk, span, d)
    v = v.view(b, -1, hk, s["page"], d).transpose(1, 2).float().reshape(b, hk, span, d)
    score = torch.matmul(s["q"].float().view(b, hk, hq // hk, d), k.transpose(2, 3)) / math.sqrt(d)
    if s["k_scale"] is not None:
        score = score * s["k_scale"][:, None, None]
    where = torch.arange(span, device=DEVICE)
    seen = where < s["lengths"][:, None]
    if s["window"]:
        seen = seen & (where >= s["lengths"][:, None] - s["window"])
    seen = seen[:, None, None, :]
    score = torch.where(seen, score, -math.inf)
    top = score.amax(3, keepdim=True)
    p = torch.where(seen, torch.exp(score - top), 0.0)
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, torch.where(seen.transpose(2, 3), v, 0.0)) / torch.where(total > 0, total, 1.0)
    if s["v_scale"] is not None:
        o = o * s["v_scale"][:, None, None]
    o = o.view(b, hq, d).to(s["q"].dtype)
    return [o, (top + total.log()).view(b, hq)] if s["lse"] else o


_run_own = {"norm": _own_norm, "matvec": _own_matvec, "append": _own_append, "attend": _own_attend}
_run_plain = {"norm": _plain_norm, "matvec": _plain_matvec, "append": _plain_append, "attend": _plain_attend}


# ---------------------------------------------------------------------------
# What a pass cannot do without.

def work(case):
    kind = case["kind"]
    if kind == "norm":
        n, e = case["rows"] * case["d"], BYTES[case["dtype"]]
        out = BYTES[_out_type(case)]
        return {"bytes": n * e * (3 if case["residual"] else 1) + n * out + case["d"] * e
                + (4 * case["rows"] if out == 1 else 0), "flops": 6 * n}
    if kind == "matvec":
        m, k, n = case["m"], case["k"], case["n"]
        return {"bytes": n * k // 2 + n * (k // case["group"]) * (3 if case["zero"] else 2) + m * k * BYTES[case["x"]]
                + m * n * BYTES[case["out"]] + (4 * m if case["x"] == "e4m3" else 0), "flops": 2 * m * k * n}
    if kind == "append":
        t, hq, hk, d = case["tokens"], case["hq"], case["hk"], case["d"]
        e, c = BYTES[case["dtype"]], BYTES[case["cache"]]
        return {"bytes": t * (2 * hq + 2 * hk) * d * e + t * 2 * hk * d * c + 12 * t + 2 * case["rot"],
                "flops": 3 * t * (hq + hk) * case["rot"]}
    b, hq, hk, d = case["batch"], case["hq"], case["hk"], case["d"]
    seen = [min(n, case["window"] or n) for n in _lengths(case)]
    pages = sum((n + case["page"] - 1) // case["page"] for n in seen)
    return {"bytes": 2 * sum(seen) * hk * d * BYTES[case["cache"]] + 2 * b * hq * d * BYTES[case["dtype"]] + 4 * pages + 4 * b
            + (4 * b * hq if case["lse"] else 0), "flops": 4 * sum(seen) * hq * d}


# ---------------------------------------------------------------------------
# The definitions in 64 bits.

def _e4m3(x):
    """The nearest e4m3 value (ties to even): 3 bits after the leading one, exponents down to -6, at most 448."""
    exponent = torch.frexp(x)[1].clamp(min=-5) - 1
    unit = torch.ldexp(torch.ones_like(x), exponent - 3)
    return (torch.round(x / unit) * unit).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "matvec": _exact_matvec, "append": _exact_append, "attend": _exact_attend}[case["kind"]](s)


def _exact_norm(s):
    h = s["x"].double()
    if s["h"] is not None:
        h += s["h"].double()
    size = torch.linalg.vector_norm(h, dim=1) ** 2 / s["d"] + s["eps"]
    y = h / size.sqrt()[:, None] * s["weight"].double()
    kept = None if s["h"] is None else h
    if s["out"] != "e4m3":
        return [y, None, kept]
    scale = torch.maximum(y.amax(1), -y.amin(1)) / E4M3_MAX
    return [_e4m3(y / scale[:, None]), scale, kept]


def _exact_matvec(s):
    x = s["x"].double()
    if s["x_scale"] is not None:
        x = x * s["x_scale"].double()[:, None]
    low, high = (s["weight"] % 16).double(), (s["weight"] // 16).double()
    half = s["group"] // 2
    y = torch.zeros(s["m"], s["n"], dtype=torch.float64, device=DEVICE)
    for i in range(s["k"] // s["group"]):
        cols = slice(i * half, (i + 1) * half)
        xs = x[:, i * s["group"]:(i + 1) * s["group"]]
        part = xs[:, 0::2].contiguous() @ low[:, cols].t().contiguous() + xs[:, 1::2].contiguous() @ high[:, cols].t().contiguous()
        zero = s["zero"][:, i].double() if s["zero"] is not None else torch.full((s["n"],), 8.0, dtype=torch.float64, device=DEVICE)
        y += (part - xs.sum(1)[:, None] * zero[None]) * s["scale"][:, i].double()[None]
    return y


def _exact_append(s):
    half, rot = s["rot"] // 2, s["rot"]
    i = torch.arange(half, device=DEVICE)
    first, second = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + half)
    angle = torch.outer(s["positions"].double(), s["inv_freq"].double())
    turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle)[:, None]

    def turned(x):
        x = x.double().clone()
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    caches = []
    for x, cache, scale in ((turned(s["k"]), s["k_cache"], s["k_scale"]), (s["v"].double(), s["v_cache"], s["v_scale"])):
        rows = cache.double().transpose(1, 2).flatten(0, 1)       # [slot, head, d]
        rows[s["slots"]] = x if scale is None else _e4m3(x / scale.double()[:, None])
        caches.append(rows.view(-1, s["page"], s["hk"], s["d"]).transpose(1, 2))
    assert rot <= s["d"]
    return [turned(s["q"]), *caches]


def _exact_attend(s):
    group, page = s["hq"] // s["hk"], s["page"]
    out = torch.zeros(s["batch"], s["hq"], s["d"], dtype=torch.float64, device=DEVICE)
    lse = torch.full((s["batch"], s["hq"]), -math.inf, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s["lengths"].tolist()):
        low = max(0, n - s["window"]) if s["window"] else 0
        if n <= low:
            continue
        at = torch.arange(low, n, device=DEVICE)
        pg, off = s["table"][b].long()[at // page], at % page
        for h in range(s["hk"]):
            eight = s["k_scale"] is not None
            k, v = ((c.view(torch.uint8)[pg, h, off].view(torch.float8_e4m3fn) if eight else c[pg, h, off]).double()
                    for c in (s["k_cache"], s["v_cache"]))
            if eight:
                k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
            rows = slice(h * group, (h + 1) * group)
            score = (k @ s["q"][b, rows].double().t().contiguous()).t() / math.sqrt(s["d"])
            lse[b, rows] = torch.logsumexp(score, 1)
            out[b, rows] = torch.softmax(score, 1) @ v
    return [out, lse] if s["lse"] else out
