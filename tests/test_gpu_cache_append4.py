"""coverprune_kv_append4 and coverprune_kv_gather against their float64 statements."""
import math

import pytest

from tests import cache_ref, serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def _data(tokens, hq, hk, d, rot, page, t, seed=0, pad=0, size=1.0, far=10):
    g = torch.Generator(device="cuda").manual_seed(seed + tokens + d)
    wide = (hq + 2 * hk) * d + pad
    qkv = (size * torch.randn(tokens, wide, device="cuda", generator=g)).to(t)
    q, k, v = (qkv[:, a * d:b * d].unflatten(1, (-1, d)) for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk)))
    pages = (tokens + page - 1) // page + 1
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:tokens]
    pos = torch.randint(0, far * max(tokens, 100), (tokens,), device="cuda", generator=g, dtype=torch.int32)
    inv = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda") / max(rot, 1)) if rot else None
    fill = dict(dtype=torch.uint8, device="cuda")
    caches = [torch.full((pages, hk, page, d // 2), 0xa5, **fill), torch.full((pages, hk, page, d // 2), 0x5a, **fill),
              torch.full((pages, hk, page, d // 32), 0x77, **fill), torch.full((pages, hk, page, d // 32), 0x78, **fill)]
    return q, k, v, pos, slots, inv, caches


def _rows(cache, slots):
    page = cache.shape[2]
    return cache.cpu()[slots // page, :, slots % page]


def _check(q, k, v, pos, slots, inv, caches, interleaved=False, magnitude=1.0):
    import paper_2608_13226_amd as cp
    before = [c.clone() for c in caches]
    t = k.dtype
    out = cp.kv_append4(q, k, v, pos, slots, inv, *caches, interleaved=interleaved, magnitude=magnitude)
    want, size = ref.rotate(q, pos, inv, interleaved, magnitude)
    # float32 rotation: two products and a sum, and sines and cosines to 2^-23.
    ref.assert_close(out, want, t, 2.0 ** -21 * size, "q")
    kd, ksize = ref.rotate(k, pos, inv, interleaved, magnitude)
    pages, page = caches[0].shape[0], caches[0].shape[2]
    s = slots.cpu()
    stored = (s >= 0) & (s < pages * page)
    for x, size, cache, scale, what in ((kd, ksize, caches[0], caches[2], "k"), (ref.d64(v), torch.zeros_like(kd), caches[1], caches[3], "v")):
        x, size = x[stored], size[stored]
        code, e = cache_ref.blocks(x, t)
        got, gote = cache_ref.unpack(_rows(cache, s[stored])), _rows(scale, s[stored]).int()
        # float64: angles, sines and products to a few of 2^-53 of the pair's size, angles of up to 2^20 to 2^-33.
        differ = (got != code) | (gote != e).repeat_interleave(32, -1)
        if bool(differ.any()):
            assert bool(cache_ref.margin(x, size * (2.0 ** -48 + 2.0 ** -52 * float(pos.abs().max())), t)[differ].all()), f"{what}: codes differ"
    # Slots that no token went to are as they were.
    used = torch.zeros(pages * page, dtype=torch.bool)
    used[s[stored]] = True
    for c, b in zip(caches, before):
        same = (c == b).all(3).cpu().transpose(1, 2).flatten(0, 1).all(1)
        assert bool(same[~used].all())
    return out


@pytest.mark.parametrize("tokens,hq,hk,d,rot,page,t,inter", [
    (1, 28, 4, 128, 128, 16, BF, False), (1, 1, 1, 32, 2, 1, F16, False), (3, 8, 8, 64, 32, 7, F16, True),
    (5, 2, 1, 96, 96, 50, BF, False), (17, 4, 2, 96, 24, 16, F16, False), (64, 7, 1, 256, 64, 64, BF, True),
    (300, 6, 3, 192, 192, 100, BF, False), (1638, 28, 4, 128, 128, 64, BF, False), (40, 3, 1, 64, 6, 16, BF, False),
    (700, 2, 2, 64, 64, 16, F16, False), (9, 5, 5, 32, 0, 4, BF, False), (33, 1, 2, 160, 100, 32, F16, True),
    (2, 2, 2, 4096, 4096, 2, BF, False)])
def test_append4(tokens, hq, hk, d, rot, page, t, inter):
    print(f"append4 {tokens} {hq}/{hk} d={d} rot={rot} {t} inter={inter}", flush=True)
    _check(*_data(tokens, hq, hk, d, rot, page, t), interleaved=inter, magnitude=1.2)


@pytest.mark.parametrize("inter", [False, True])
def test_rows_without_alignment(inter):
    q, k, v, pos, slots, inv, caches = _data(19, 4, 2, 64, 32, 16, BF, pad=3)
    _check(q, k, v, pos, slots, inv, caches, interleaved=inter)


def test_without_queries_and_slots_outside():
    import paper_2608_13226_amd as cp
    q, k, v, pos, slots, inv, caches = _data(40, 4, 2, 128, 128, 16, BF)
    slots[::3] = -1
    slots[1] = caches[0].shape[0] * 16
    slots[4] = 2 ** 62
    _check(q, k, v, pos, slots, inv, caches)
    again = [torch.full_like(c, 1) for c in caches]
    for c, a in zip(caches, again):
        a.copy_(c)
    assert cp.kv_append4(None, k, v, pos, slots, inv, *again) is None
    assert all(torch.equal(a, c) for a, c in zip(again, caches))


@pytest.mark.parametrize("t", [BF, F16])
@pytest.mark.parametrize("far", [1 << 20, 20_000_000])
def test_far_positions(t, far):
    q, k, v, pos, slots, inv, caches = _data(100, 4, 4, 128, 128, 16, t, far=far // 100)
    pos[0], pos[1] = -7, 0
    _check(q, k, v, pos, slots, inv, caches)


@pytest.mark.parametrize("t", [BF, F16])
def test_borders_zeros_and_ends_of_the_range(t):
    """Ties, blocks whose largest is at 6 times a power or next to it, zeros, -0, subnormal and largest numbers."""
    low, high = cache_ref.POWERS[t]
    info = torch.finfo(t)
    rows = []
    for e in (0, -3, 4, low, low - 1, low - 2, high, high - 1):
        base = torch.tensor([0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, .5, 1, 1.5, 2, 3, 4, .2500001], dtype=torch.float64) * 2.0 ** max(e, -140)
        rows.append(torch.cat([base, -base]))
        rows.append(torch.cat([base.clamp(max=5 * 2.0 ** max(e, -140)), -base.clamp(max=3 * 2.0 ** max(e, -140))]))
    six = torch.tensor(6.0, dtype=t)
    near = [six, torch.nextafter(six.float(), torch.tensor(9.0)).to(t), (six.double() * (1 + info.eps)).to(t), (six.double() * (1 - info.eps)).to(t)]
    rows += [torch.cat([torch.full((1,), float(n), dtype=torch.float64), torch.linspace(-5, 5, 31, dtype=torch.float64)]) for n in near]
    rows += [torch.zeros(32, dtype=torch.float64), torch.full((32,), -0.0, dtype=torch.float64),
             torch.full((32,), info.max, dtype=torch.float64), torch.full((32,), -info.max, dtype=torch.float64),
             torch.full((32,), info.smallest_normal, dtype=torch.float64), torch.full((32,), info.smallest_normal * info.eps, dtype=torch.float64)]
    x = torch.stack(rows).to(t).cuda()
    n = x.shape[0]
    caches = [torch.zeros(n, 1, 1, w, dtype=torch.uint8, device="cuda") for w in (16, 16, 1, 1)]
    _check(x[:, None].contiguous(), x[:, None], x[:, None], torch.zeros(n, dtype=torch.int32, device="cuda"),
           torch.arange(n, device="cuda"), None, caches)
    held = cache_ref.values(caches[1], caches[3])
    assert bool(torch.isfinite(held).all()) and bool(torch.isfinite(held.to(t)).all())
    # Every value that is held is one of the type.
    assert torch.equal(held.to(t).double(), held)


@pytest.mark.parametrize("t", [BF, F16])
def test_infinities_and_nan_take_their_block_alone(t):
    import paper_2608_13226_amd as cp
    q, k, v, pos, slots, inv, caches = _data(6, 2, 2, 128, 64, 16, t)
    k, v = k.clone(), v.clone()
    k[0, 0, 5], k[1, 1, 70], k[2, 0, 127], v[3, 1, 0], v[4, 0, 33] = math.inf, -math.inf, math.nan, math.nan, math.inf
    cp.kv_append4(None, k, v, pos, slots, inv, *caches)
    kd, _ = ref.rotate(k, pos, inv, False, 1.0)
    for x, cache, scale in ((kd, caches[0], caches[2]), (ref.d64(v), caches[1], caches[3])):
        bad = ~torch.isfinite(x.unflatten(-1, (-1, 32))).all(-1)
        e = _rows(scale, slots.cpu())
        assert torch.equal(e == 255, bad) and int(bad.sum()) >= 2
        assert not bool(_rows(cache, slots.cpu()).unflatten(-1, (-1, 16))[bad].any())


def test_keys_past_float32_saturate():
    """Rotated and enlarged past float32's range, with finite inputs."""
    q, k, v, pos, slots, inv, caches = _data(4, 1, 1, 64, 64, 16, BF)
    k = torch.full_like(k, torch.finfo(BF).max)
    _check(q, k, v, pos, slots, inv, caches, magnitude=3.0)
    assert bool((_rows(caches[2], slots.cpu()) == 252).all())


@pytest.mark.parametrize("t", [BF, F16])
@pytest.mark.parametrize("inter", [False, True])
def test_magnitude_is_taken_in_64_bits(t, inter):
    """1.2 * 5 is 6 in float64, where a block keeps its power; with 1.2 rounded to float32, 4e-8 too large, it would be past it."""
    import paper_2608_13226_amd as cp
    assert 1.2 * 5 == 6.0 and 1.2 * 1.25 == 1.5 and 5 * float(torch.tensor(1.2)) > 6.0
    q, k, v, pos, slots, inv, caches = _data(3, 1, 1, 32, 32, 16, t)
    k = torch.full_like(k, 1.25)
    k[:, :, 0] = 5.0
    pos.zero_()
    cp.kv_append4(None, k, v, pos, slots, inv, *caches, interleaved=inter, magnitude=1.2)
    assert bool((_rows(caches[2], slots.cpu()) == 127).all())
    codes = cache_ref.unpack(_rows(caches[0], slots.cpu()))
    assert bool((codes[..., 0] == 7).all()) and bool((codes[..., 1:] == 3).all())


def test_no_tokens():
    import paper_2608_13226_amd as cp
    q, k, v, pos, slots, inv, caches = _data(0, 2, 1, 64, 64, 16, BF)
    assert cp.kv_append4(q, k, v, pos, slots, inv, *caches).shape == (0, 2, 64)
    a, b = cp.kv_gather(caches[0], caches[1], slots, k_scale=caches[2], v_scale=caches[3])
    assert a.shape == b.shape == (0, 1, 64)


# ---------------------------------------------------------------------------
# Reading rows back.

@pytest.mark.parametrize("held", ["same", "e4m3", "e2m1"])
@pytest.mark.parametrize("tokens,hk,d,page,t", [(1, 1, 32, 1, BF), (5, 4, 128, 16, BF), (1000, 2, 96, 50, F16), (77, 16, 64, 7, BF),
                                                (300, 1, 256, 128, F16), (9, 3, 20, 8, BF), (4, 1, 1, 3, F16)])
def test_gather(tokens, hk, d, page, t, held):
    import paper_2608_13226_amd as cp
    if held == "e2m1" and d % 32:
        pytest.skip("4-bit rows are of 32 dims")
    print(f"gather {tokens} {hk} d={d} page={page} {t} {held}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(tokens + d)
    pages = (tokens + page - 1) // page + 2
    slots = torch.randint(0, pages * page, (tokens,), device="cuda", generator=g)      # some twice
    if tokens > 3:
        slots[0], slots[3] = -5, pages * page
    caches, scales = [], []
    for _ in range(2):
        if held == "e2m1":
            caches.append(torch.randint(0, 256, (pages, hk, page, d // 2), device="cuda", generator=g, dtype=torch.uint8))
            # Exponents that the type holds with all codes, and the one without a value.
            low, high = cache_ref.POWERS[t]
            e = torch.randint(low + 127, high + 128, (pages, hk, page, d // 32), device="cuda", generator=g).to(torch.uint8)
            scales.append(torch.where(torch.rand(e.shape, device="cuda", generator=g) < 0.1, torch.full_like(e, 255), e))
        else:
            x = torch.randn(pages, hk, page, d, device="cuda", generator=g)
            caches.append((100 * x).clamp(-448, 448).to(E4M3) if held == "e4m3" else x.to(t))
            scales.append(0.01 + torch.rand(hk, device="cuda", generator=g) if held == "e4m3" else None)
    got = cp.kv_gather(*caches, slots, dtype=t, k_scale=scales[0], v_scale=scales[1])
    s = slots.cpu()
    inside = (s >= 0) & (s < pages * page)
    at = torch.where(inside, s, torch.zeros_like(s))
    for x, cache, scale in zip(got, caches, scales):
        if held == "e2m1":
            want = cache_ref.values(cache, scale)[at // page, :, at % page]
        else:
            want = ref.d64(cache)[at // page, :, at % page]
            if held == "e4m3":
                want = want * ref.d64(scale)[:, None]
        want = torch.where(inside[:, None, None], want, torch.zeros_like(want))
        assert x.dtype == t and x.shape == want.shape
        if held == "e4m3":
            ref.assert_close(x, want, t, 2.0 ** -24 * want.abs(), "row")       # a float32 product, then the rounding
        else:
            assert torch.equal(torch.nan_to_num(ref.d64(x), nan=1e300), torch.nan_to_num(want, nan=1e300))


def test_gather_of_e4m3_without_scales_and_nan():
    import paper_2608_13226_amd as cp
    codes = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(1, 1, 8, 32).cuda()
    cache = codes.view(E4M3)
    k, v = cp.kv_gather(cache, cache, torch.arange(8, device="cuda"))
    want = ref.d64(cache)[0, 0]
    assert torch.equal(torch.nan_to_num(ref.d64(k)[:, 0], nan=1e9), torch.nan_to_num(want, nan=1e9)) and k.dtype == BF


def test_append_then_gather_gives_the_values_back():
    """What is exact in 4 bits comes back as it went in."""
    import paper_2608_13226_amd as cp
    g = torch.Generator(device="cuda").manual_seed(0)
    level = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device="cuda")[torch.randint(0, 8, (50, 3, 64), device="cuda", generator=g)]
    level[..., 0], level[..., 32] = 6, 6
    x = (level * torch.where(torch.rand(level.shape, device="cuda", generator=g) < 0.5, -0.25, 0.25)).to(F16)
    caches = [torch.zeros(10, 3, 8, w, dtype=torch.uint8, device="cuda") for w in (32, 32, 2, 2)]
    slots = torch.randperm(80, device="cuda", generator=g)[:50]
    cp.kv_append4(None, x, -x, torch.zeros(50, dtype=torch.int32, device="cuda"), slots, None, *caches)
    k, v = cp.kv_gather(caches[0], caches[1], slots, F16, caches[2], caches[3])
    assert torch.equal(k, x) and torch.equal(v, -x)
