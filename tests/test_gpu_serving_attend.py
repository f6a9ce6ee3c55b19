"""coverprune_paged_attention against its float64 statement."""
import math

import pytest

from tests import serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def _data(lengths, hq, hk, d, page, t, c, seed=0, sharp=1.0, garbage=True):
    g = torch.Generator(device="cuda").manual_seed(seed + hq + d + page + len(lengths))
    b = len(lengths)
    width = max(1, (max(lengths) + page - 1) // page)
    pages = b * width + 2
    eight = c == E4M3

    def cache():
        x = torch.randn(pages, hk, page, d, device="cuda", generator=g)
        return (60.0 * x).clamp(-448, 448).to(E4M3) if eight else x.to(c)

    k, v = cache(), cache()
    table = torch.randperm(pages, device="cuda", generator=g)[:b * width].view(b, width).to(torch.int32)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if garbage:
        # Every slot that holds no token: NaN, infinities and the lowest values.
        used = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
        at = torch.arange(width * page, device="cuda")
        for i in range(b):
            used[table[i].long()[at // page][:lengths[i]], (at % page)[:lengths[i]]] = True
        bits = torch.uint8 if eight else torch.int16
        # e4m3: NaN and +-448; bf16 and f16: NaN, -inf, and about the lowest finite value.
        if eight:
            junk = torch.tensor([0x7f, 0xff, 0x7e, 0xfe], dtype=torch.int16, device="cuda").to(torch.uint8)
        else:
            info = torch.finfo(c)
            junk = torch.tensor([math.nan, -math.inf, math.inf, info.min], device="cuda").to(c).view(bits)
        fill = junk[torch.arange(pages * page, device="cuda") % 4].view(pages, 1, page, 1).expand(pages, hk, page, d)
        for x in (k, v):
            raw = x.view(bits)
            raw.copy_(torch.where(used[:, None, :, None], raw, fill))
        table = torch.where(torch.arange(width, device="cuda") * page < n[:, None], table, torch.full_like(table, 2 ** 31 - 1))
    q = (sharp * torch.randn(b, hq, d, device="cuda", generator=g)).to(t)
    ks = (0.005 + 0.02 * torch.rand(hk, device="cuda", generator=g)) if eight else None
    vs = (0.005 + 0.02 * torch.rand(hk, device="cuda", generator=g)) if eight else None
    return dict(q=q, k_cache=k, v_cache=v, table=table, lengths=n, k_scale=ks, v_scale=vs)


def _check(a, window=0, scale=None, max_length=None, **kw):
    import paper_2608_13226_amd as cp
    if max_length is None:
        max_length = max(1, int(a["lengths"].max()))
    out, lse = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], max_length=max_length,
                                  window=window, scale=scale, k_scale=a["k_scale"], v_scale=a["v_scale"], return_lse=True, **kw)
    want, wlse, size = ref.attend(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], window, scale, a["k_scale"],
                                  a["v_scale"])
    # Scores: d products summed in float32, exponentials of them, sums of p and p v; all are within
    # 2^-24 (d + tokens / 32 + 100) of the summands' sizes, and scores here are below 60.
    tokens = int(a["lengths"].max())
    d = a["q"].shape[2]
    work = 2.0 ** -24 * (60 * (d / 32 + 8) + tokens / 32 + 100)
    ref.assert_close(out, want, out.dtype, work * size, "out")
    ref.assert_close(lse, wlse, torch.float32, work * (1 + torch.where(torch.isfinite(wlse), wlse.abs(), torch.zeros_like(wlse))), "lse")
    return out, lse


@pytest.mark.parametrize("c8", [False, True])
@pytest.mark.parametrize("lengths,hq,hk,d,page,t", [
    ([1], 1, 1, 64, 16, BF), ([1, 0, 2], 28, 4, 128, 16, BF), ([31, 32, 33, 64, 65], 16, 16, 64, 50, F16),
    ([629], 28, 4, 128, 16, BF), ([5, 300, 1000, 0, 77], 8, 1, 256, 7, F16), ([513, 200], 20, 1, 96, 1, BF),
    ([4096, 3], 12, 12, 192, 100, BF), ([1500, 1501, 1503], 32, 2, 128, 64, F16), ([130], 40, 2, 64, 128, BF),
    ([2500], 6, 2, 96, 32, F16), ([700, 1], 34, 1, 192, 33, F16)])
def test_attention(lengths, hq, hk, d, page, t, c8):
    print(f"attend lengths={lengths} heads={hq}/{hk} d={d} page={page} {t} c8={c8}", flush=True)
    _check(_data(lengths, hq, hk, d, page, t, E4M3 if c8 else t))


@pytest.mark.parametrize("window", [1, 31, 32, 100, 640, 5000])
def test_window(window):
    a = _data([0, 1, 33, 700, 2100], 8, 2, 128, 16, BF, BF)
    _check(a, window=window)
    _check(a, window=window, max_length=a["table"].shape[1] * 16)


def test_no_tokens_at_all():
    import paper_2608_13226_amd as cp
    a = _data([0, 0, 0], 8, 2, 128, 16, BF, BF)
    out, lse = _check(a)
    assert not bool(out.any()) and bool(torch.isneginf(lse).all())
    _check(a, max_length=16)
    a = _data([64], 8, 2, 128, 16, BF, BF)
    empty = cp.paged_attention(a["q"][:0], a["k_cache"], a["v_cache"], a["table"][:0], a["lengths"][:0], max_length=64)
    assert empty.shape == (0, 8, 128)


def test_lengths_are_held_to_what_the_host_said():
    """Lengths over max_length count as max_length, negative ones as 0."""
    a = _data([300, 200], 8, 2, 128, 16, BF, BF, garbage=False)
    import paper_2608_13226_amd as cp
    b = dict(a, lengths=torch.tensor([250, 0], dtype=torch.int32, device="cuda"))
    want, wl = _check(b, max_length=250)
    got, gl = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"],
                                 torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32, device="cuda"), max_length=250, return_lse=True)
    assert torch.equal(got, want) and torch.equal(gl, wl)


@pytest.mark.parametrize("c8", [False, True])
def test_sharp_scores(c8):
    """One token far above all others, early or late in the run: the maximum moves, and the rest underflows."""
    a = _data([1200, 1200, 40], 8, 2, 128, 16, BF, E4M3 if c8 else BF, sharp=0.05, garbage=False)
    for b, at in ((0, 3), (1, 1190), (2, 39)):
        page, off = int(a["table"][b, at // 16]), at % 16
        for h in range(2):
            row = 3.0 * a["q"][b, 4 * h].float() / 0.05
            a["k_cache"][page, h, off] = (row * 60).clamp(-448, 448).to(E4M3) if c8 else row.to(BF)
    _check(a, scale=0.5)


def test_scales_of_any_sign_and_zero():
    a = _data([333], 8, 2, 64, 16, F16, F16)
    _check(a, scale=0.0)
    _check(a, scale=-0.25)


def test_bad_values_among_the_tokens_stay_in_their_sequence():
    import paper_2608_13226_amd as cp
    a = _data([500, 500], 8, 2, 128, 16, BF, BF, garbage=False)
    clean = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], max_length=500)
    a["v_cache"][int(a["table"][0, 3]), 1, 5, 7] = math.nan
    got = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], max_length=500)
    assert torch.equal(got[1], clean[1]) and torch.equal(got[0, :4], clean[0, :4])
    assert bool(torch.isnan(got[0, 4:, 7]).all())
    rest = [i for i in range(128) if i != 7]
    assert torch.equal(got[0, 4:][:, rest], clean[0, 4:][:, rest])


def test_a_long_sequence_and_its_pieces():
    """Joining two halves by their lse gives the whole."""
    import paper_2608_13226_amd as cp
    a = _data([40000], 28, 4, 128, 64, BF, BF)
    whole, lse = _check(a)
    half = 64 * 313
    kw = dict(return_lse=True)
    o1, l1 = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], torch.tensor([half], dtype=torch.int32, device="cuda"),
                                max_length=half, **kw)
    o2, l2 = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"][:, 313:].contiguous(),
                                torch.tensor([40000 - half], dtype=torch.int32, device="cuda"), max_length=40000 - half, **kw)
    w = torch.softmax(torch.stack([l1, l2]), 0)[..., None]
    both = o1.float() * w[0] + o2.float() * w[1]
    assert float((both - whole.float()).abs().max()) <= 2.0 ** -7 * float(whole.float().abs().max())
    assert float((torch.logaddexp(l1, l2) - lse).abs().max()) < 1e-4


def test_a_cache_past_32_bits():
    """Pages whose byte offset does not fit 32 bits, and neither do their rows a signed one."""
    import paper_2608_13226_amd as cp
    page, hk, d = 64, 8, 64
    pages = 2 ** 31 // (page * hk) + 1000                       # over 2^31 rows of 64 bytes: 128 GiB a cache
    free, _ = torch.cuda.mem_get_info()
    if free < 2 * pages * page * hk * d + (8 << 30):
        pytest.skip("not enough free memory on this card")
    k = torch.empty(pages, hk, page, d, device="cuda", dtype=torch.uint8).view(E4M3)
    v = torch.empty(pages, hk, page, d, device="cuda", dtype=torch.uint8).view(E4M3)
    small = _data([70], 16, hk, d, page, BF, E4M3, garbage=False)
    mine = torch.tensor([[pages - 1, pages - 500]], dtype=torch.int32, device="cuda")
    for big, s in ((k, small["k_cache"]), (v, small["v_cache"])):
        for i in range(2):
            big.view(torch.uint8)[int(mine[0, i])] = s.view(torch.uint8)[int(small["table"][0, i])]
    kw = dict(max_length=70, k_scale=small["k_scale"], v_scale=small["v_scale"])
    got = cp.paged_attention(small["q"], k, v, mine, small["lengths"], **kw)
    want = cp.paged_attention(small["q"], small["k_cache"], small["v_cache"], small["table"], small["lengths"], **kw)
    assert torch.equal(got, want)
    del k, v
    torch.cuda.empty_cache()


def test_the_same_answer_every_time_and_any_workspace():
    import paper_2608_13226_amd as cp
    lib = cp.library()
    a = _data([9000, 20, 4000], 28, 4, 128, 16, BF, BF)
    out, lse = _check(a)
    need = lib.coverprune_paged_attention_workspace(3, 28, 4, 128, 9000, 0)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")      # NaN everywhere
    for _ in range(3):
        o, s = _check(a, workspace=ws)
        assert torch.equal(o, out) and torch.equal(s, lse)
    if need:
        with pytest.raises(cp.CoverPruneError, match="workspace"):
            cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], max_length=9000,
                               workspace=ws[:need - 64])


@pytest.mark.parametrize("c8", [False, True])
@pytest.mark.parametrize("page", [16, 32])
@pytest.mark.parametrize("t", [F16, BF])
def test_weights_far_below_the_largest(t, page, c8):
    """A token of each 32 has exp(18) times the others' weight and no value: what the others give is the result."""
    import paper_2608_13226_amd as cp
    n, d = 64, 64
    a = _data([n], 8, 2, d, page, t, E4M3 if c8 else t, garbage=False)
    a["k_scale"] = a["v_scale"] = None
    a["q"] = torch.ones_like(a["q"])
    g = torch.Generator().manual_seed(5)
    keys = torch.zeros(n, 1, 1).expand(n, 2, d).clone()
    keys[5::32] = 18.0 / d
    values = 200.0 + 200.0 * torch.rand(n, 2, d, generator=g)
    values[5::32] = 0.0
    at = torch.arange(n, device="cuda")
    pages, off = a["table"][0].long()[at // page], at % page
    c = a["k_cache"].dtype
    for cache, x in ((a["k_cache"], keys), (a["v_cache"], values)):
        cache.view(torch.uint8).view(*cache.shape[:3], -1)[pages, :, off] = x.to(c).cuda().view(torch.uint8)
    out, lse = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], scale=1.0, return_lse=True)
    want, wlse, size = ref.attend(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], 0, 1.0)
    # float16 holds a weight to 2^-36 of the largest; the rest is float32 work (bfloat16: two parts, 2^-16).
    ref.assert_close(out, want, t, 2.0 ** -16 * size + n * 2.0 ** -36 * 448.0 * (t == F16), "out")
    ref.assert_close(lse, wlse, torch.float32, 2.0 ** -18 * wlse.abs(), "lse")


@pytest.mark.parametrize("t", [F16, BF])
@pytest.mark.parametrize("shut", [0, 1, 32, 33, 64, 700, 3000])
def test_scores_of_minus_infinity_count_nothing(shut, t):
    """Keys that rule their tokens out, whole tiles and runs of them; the values there are ordinary."""
    import paper_2608_13226_amd as cp
    a = _data([3001, 0], 8, 2, 64, 16, t, t, garbage=False)
    a["q"][:, :, 0] = 1.0
    at = torch.arange(shut, device="cuda")
    a["k_cache"][a["table"][0].long()[at // 16], :, at % 16, 0] = -math.inf
    _check(a)
    at = torch.arange(3001, device="cuda")
    a["k_cache"][a["table"][0].long()[at // 16], :, at % 16, 0] = -math.inf
    out, lse = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], max_length=3001, return_lse=True)
    assert not bool(out.any()) and bool(torch.isneginf(lse).all())


@pytest.mark.parametrize("c8", [False, True])
@pytest.mark.parametrize("t", [F16, BF])
@pytest.mark.parametrize("n,d,page", [(2, 64, 16), (2, 128, 32), (64, 96, 50), (700, 128, 64), (900, 192, 16)])
def test_weights_keep_float32s_bits(n, d, page, t, c8):
    """Values of 1 and -1 in turn under nearly equal weights: what is left of their sum shows the weights' last bits."""
    import paper_2608_13226_amd as cp
    a = _data([n] * 32, 28, 4, d, page, t, E4M3 if c8 else t, garbage=False)
    a["k_scale"] = a["v_scale"] = None
    g = torch.Generator(device="cuda").manual_seed(n + d)
    a["q"].zero_()
    a["q"][:, :, 0] = 1.0 + torch.rand(32, 28, device="cuda", generator=g).to(t)
    c = a["k_cache"].dtype
    at = torch.arange(n, device="cuda")
    keys = torch.zeros(n, 4, d, device="cuda")
    keys[:, :, 0] = torch.randint(1, 8, (n, 4), device="cuda", generator=g) * 2.0 ** -9
    keys[1, :, 0] = 0.0
    values = (1.0 - 2.0 * (at % 2))[:, None, None].expand(n, 4, d)
    for b in range(32):
        pages, off = a["table"][b].long()[at // page], at % page
        for cache, x in ((a["k_cache"], keys), (a["v_cache"], values)):
            cache.view(torch.uint8).view(*cache.shape[:3], -1)[pages, :, off] = x.contiguous().to(c).view(torch.uint8)
    scale = 2.0 ** -6
    out = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], max_length=n, scale=scale)
    want, _, size = ref.attend(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], 0, scale)
    # Scores below 2^-10, so a weight is an exponential's 2^-23 off and no more; sums of n / 32 steps a wave, at
    # most 2^-24 (n / 128 + 8) of the summands' size.
    ref.assert_close(out, want, t, 2.0 ** -20 * size, "out")


@pytest.mark.parametrize("t", [F16, BF])
@pytest.mark.parametrize("lengths,hq,hk,d,page", [([1, 2], 4, 2, 64, 16), ([33, 5], 28, 4, 128, 50), ([700, 1500], 8, 2, 96, 32),
                                                  ([4000], 6, 1, 256, 64)])
def test_infinite_values_among_the_tokens(lengths, hq, hk, d, page, t):
    """An infinite value makes its dimension infinite, two of both signs NaN; all else stays."""
    a = _data(lengths, hq, hk, d, page, t, t, seed=2)
    for b, n in enumerate(lengths):
        for i, (at, dim, value) in enumerate([(0, 3, math.inf), (n - 1, 7, -math.inf), (n // 2, d - 1, math.inf),
                                              (0, 20, math.inf), (n - 1, 20, -math.inf if n > 1 else math.inf)]):
            a["v_cache"][int(a["table"][b, at // page]), i % hk, at % page, dim] = value
            if i >= 3:
                a["v_cache"][int(a["table"][b, at // page]), :, at % page, dim] = value
    out, _ = _check(a)
    assert bool(torch.isinf(out).any()) and bool(torch.isnan(out).any()) == (max(lengths) > 1)


@pytest.mark.parametrize("t", [F16, BF])
def test_one_token_is_its_value(t):
    """The only token's weight is 1, whatever its value."""
    import paper_2608_13226_amd as cp
    a = _data([1], 8, 2, 64, 16, t, t)
    row = a["v_cache"][int(a["table"][0, 0]), :, 0]
    row[0, :6] = torch.tensor([math.inf, -math.inf, math.nan, torch.finfo(t).max, torch.finfo(t).min, torch.finfo(t).tiny], dtype=t)
    out = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], max_length=1)
    want = row.repeat_interleave(4, 0)[None]
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(out), nan) and torch.equal(out[~nan], want[~nan])


@pytest.mark.parametrize("n", [280, 5000])
def test_values_near_the_end_of_float32(n):
    """Two tokens of a wave, the later one's weight 148 times the first's: no sum passes float32's range."""
    a = _data([n], 8, 2, 128, 16, BF, BF, garbage=False)
    a["q"] = torch.ones_like(a["q"])
    at = torch.arange(n, device="cuda")
    pages, off = a["table"][0].long()[at // 16], at % 16
    keys = torch.full((n, 2, 128), -0.25, device="cuda")
    values = torch.ones(n, 2, 128, device="cuda")
    for at, score, value in ((3, 0.0, 1e38), (260, 5.0, 2e38)):
        keys[at], values[at] = 0.0, value
        keys[at, :, 0] = score
    for cache, x in ((a["k_cache"], keys), (a["v_cache"], values)):
        cache[pages, :, off] = x.to(BF)
    out, _ = _check(a, scale=1.0)
    assert bool(torch.isfinite(out).all())
