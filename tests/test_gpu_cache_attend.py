"""coverprune_paged_attention4 and coverprune_paged_attention_mass against their float64 statements."""
import math

import pytest

from tests import cache_ref, serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def _data(lengths, hq, hk, d, page, t, held="e2m1", seed=0, sharp=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + hq + d + page + len(lengths))
    b = len(lengths)
    width = max(1, (max(lengths) + page - 1) // page)
    pages = b * width + 2
    table = torch.randperm(pages, device="cuda", generator=g)[:b * width].view(b, width).to(torch.int32)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    used = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    at = torch.arange(width * page, device="cuda")
    for i in range(b):
        used[table[i].long()[at // page][:lengths[i]], (at % page)[:lengths[i]]] = True
    used = used[:, None, :, None]
    caches, scales = [], []
    for _ in range(2):
        x = torch.randn(pages, hk, page, d, device="cuda", generator=g)
        if held == "e2m1":
            codes, e = cache_ref.cut_cache(x, t)
            # Slots that hold no token: all codes, blocks that are NaN.
            caches.append(torch.where(used, codes, torch.full_like(codes, 0x7f)))
            scales.append(torch.where(used, e, torch.full_like(e, 255)))
        elif held == "e4m3":
            codes = (60.0 * x).clamp(-448, 448).to(E4M3).view(torch.uint8)
            caches.append(torch.where(used, codes, torch.full_like(codes, 0x7f)).view(E4M3))
            scales.append(0.005 + 0.02 * torch.rand(hk, device="cuda", generator=g))
        else:
            caches.append(torch.where(used, x, torch.full_like(x, math.nan)).to(t))
            scales.append(None)
    table = torch.where(torch.arange(width, device="cuda") * page < n[:, None], table, torch.full_like(table, 2 ** 31 - 1))
    q = (sharp * torch.randn(b, hq, d, device="cuda", generator=g)).to(t)
    return dict(q=q, k_cache=caches[0], v_cache=caches[1], table=table, lengths=n, k_scale=scales[0], v_scale=scales[1])


def _work(a):
    # Scores: d products summed in float32, exponentials of them, sums of p and p v; all are within
    # 2^-24 (d + tokens / 32 + 100) of the summands' sizes, and scores here are below 60.
    return 2.0 ** -24 * (60 * (a["q"].shape[2] / 32 + 8) + int(a["lengths"].max()) / 32 + 100)


def _check_out(a, out, lse, want, wlse, size):
    ref.assert_close(out, want, out.dtype, _work(a) * size, "out")
    ref.assert_close(lse, wlse, torch.float32, _work(a) * (1 + torch.where(torch.isfinite(wlse), wlse.abs(), torch.zeros_like(wlse))), "lse")


def _check4(a, window=0, scale=None, **kw):
    import paper_2608_13226_amd as cp
    kw.setdefault("max_length", max(1, int(a["lengths"].max())))
    out, lse = cp.paged_attention4(a["q"], a["k_cache"], a["v_cache"], a["k_scale"], a["v_scale"], a["table"], a["lengths"],
                                   window=window, scale=scale, return_lse=True, **kw)
    want, wlse, size, _ = cache_ref.attend(**a, window=window, scale=scale)
    _check_out(a, out, lse, want, wlse, size)
    return out, lse


def _check_mass(a, window=0, scale=None, span=None, start=None, **kw):
    import paper_2608_13226_amd as cp
    longest = max(1, int(a["lengths"].max()))
    kw.setdefault("max_length", longest)
    batch, hk = a["q"].shape[0], a["k_cache"].shape[1]
    span = longest if span is None else span
    g = torch.Generator(device="cuda").manual_seed(5)
    mass = torch.rand(batch, hk, span, device="cuda", generator=g) if start is None else start
    before = mass.clone()
    out, lse = cp.paged_attention_mass(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], mass, window=window, scale=scale,
                                       k_scale=a["k_scale"], v_scale=a["v_scale"], return_lse=True, **kw)
    want, wlse, size, more = cache_ref.attend(**a, window=window, scale=scale)
    _check_out(a, out, lse, want, wlse, size)
    # A weight is off by its exponent's error (twice: in itself and in the sum), the float32 sum over the heads of a
    # group by a rounding each, and the last addition by the rounding of its result.
    added = torch.zeros(batch, hk, span, dtype=torch.float64)
    added[:, :, :more.shape[2]] = more
    group = a["q"].shape[1] // hk
    ref.assert_close(mass, ref.d64(before) + added, torch.float32, (2 * _work(a) + group * 2.0 ** -23) * added, "mass")
    # Tokens outside the sequences and windows have what they had.
    n = a["lengths"].cpu()[:, None, None]
    at = torch.arange(span)
    outside = ((at >= n) | ((at < n - window) if window else torch.zeros_like(at >= n))).expand(batch, hk, span)
    assert torch.equal(mass.cpu()[outside], before.cpu()[outside])
    return out, lse, mass


SHAPES = [([1], 1, 1, 64, 16, BF), ([1, 0, 2], 28, 4, 128, 16, BF), ([31, 32, 33, 64, 65], 16, 16, 64, 50, F16),
          ([629], 28, 4, 128, 16, BF), ([5, 300, 1000, 0, 77], 8, 1, 256, 7, F16), ([513, 200], 20, 1, 96, 1, BF),
          ([2100, 3], 12, 12, 192, 100, BF), ([1500, 1501, 1503], 32, 2, 128, 64, F16), ([130], 40, 2, 64, 128, BF),
          ([2500], 6, 2, 96, 32, F16), ([700, 1], 34, 1, 192, 33, F16)]


@pytest.mark.parametrize("lengths,hq,hk,d,page,t", SHAPES)
def test_attention4(lengths, hq, hk, d, page, t):
    print(f"attend4 lengths={lengths} heads={hq}/{hk} d={d} page={page} {t}", flush=True)
    _check4(_data(lengths, hq, hk, d, page, t))


@pytest.mark.parametrize("held", ["same", "e4m3", "e2m1"])
@pytest.mark.parametrize("lengths,hq,hk,d,page,t", SHAPES)
def test_mass(lengths, hq, hk, d, page, t, held):
    print(f"mass lengths={lengths} heads={hq}/{hk} d={d} page={page} {t} {held}", flush=True)
    a = _data(lengths, hq, hk, d, page, t, held)
    out, lse, _ = _check_mass(a)
    import paper_2608_13226_amd as cp
    longest = max(lengths)
    if held == "e2m1":
        same = cp.paged_attention4(a["q"], a["k_cache"], a["v_cache"], a["k_scale"], a["v_scale"], a["table"], a["lengths"],
                                   max_length=longest, return_lse=True)
    else:
        same = cp.paged_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], max_length=longest,
                                  k_scale=a["k_scale"], v_scale=a["v_scale"], return_lse=True)
    assert torch.equal(out, same[0]) and torch.equal(lse, same[1])


@pytest.mark.parametrize("held", ["same", "e2m1"])
@pytest.mark.parametrize("lengths,hq,hk,d,page,t", [
    ([512, 40], 16, 1, 256, 16, BF), ([500], 8, 1, 256, 50, F16), ([1024 - 25 * i for i in range(40)], 4, 2, 64, 16, BF),
    ([1000 - 10 * i for i in range(33)], 32, 2, 128, 32, F16), ([768, 760, 1], 8, 8, 128, 16, BF), ([769], 16, 1, 96, 16, F16),
    ([700], 17, 1, 64, 64, BF), ([300], 100, 2, 128, 16, BF)])
def test_mass_where_one_block_has_all_and_where_not_quite(lengths, hq, hk, d, page, t, held):
    """Scores that fit a block's LDS, or just do not; more heads than a block has columns."""
    print(f"mass {len(lengths)} sequences, heads={hq}/{hk} d={d} {t} {held}", flush=True)
    a = _data(lengths, hq, hk, d, page, t, held)
    _check_mass(a)
    _check_mass(a, window=200, span=1100)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("window", [1, 31, 33, 500, 5000])
def test_windows(window, page):
    lengths = [1, 40, 500, 0, 3001]
    print(f"window {window} page {page}", flush=True)
    _check4(_data(lengths, 8, 2, 128, page, BF), window=window)
    for held in ("same", "e2m1"):
        _check_mass(_data(lengths, 8, 2, 128, page, F16, held), window=window, span=3100)


@pytest.mark.parametrize("held", ["same", "e4m3", "e2m1"])
def test_sharp_scores_and_other_scales(held):
    # Scores spread over hundreds (below the 60 of the bound times 16).
    a = _data([300, 2000], 8, 2, 64, 32, BF, held, sharp=4.0)
    _check_mass(a, scale=0.2)
    _check_mass(a, scale=0.0)
    _check_mass(a, scale=-0.1)


def test_default_and_larger_max_length():
    a = _data([100, 1030], 4, 2, 64, 16, BF)
    out, lse = _check4(a)
    out2, lse2 = _check4(a, max_length=None)
    for x in (1040, 1031):
        _check_mass(a, span=1040, max_length=x)
    _check_mass(a, span=1037, max_length=None)
    assert torch.isfinite(out2).all()


@pytest.mark.parametrize("held", ["same", "e4m3", "e2m1"])
def test_lengths_past_max_length_and_below_zero(held):
    import paper_2608_13226_amd as cp
    a = _data([200, 90, 10], 4, 1, 128, 16, BF, held)
    b = dict(a, lengths=torch.tensor([100, 0, 10], dtype=torch.int32, device="cuda"))
    given = torch.tensor([200, -3, 10], dtype=torch.int32, device="cuda")
    results = []
    for lengths in (b["lengths"], given):
        mass = torch.zeros(3, 1, 150, device="cuda")
        out = cp.paged_attention_mass(a["q"], a["k_cache"], a["v_cache"], a["table"], lengths, mass, max_length=100, k_scale=a["k_scale"],
                                      v_scale=a["v_scale"])
        results.append((out, mass))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    assert not bool(results[0][1][:, :, 100:].any()) and not bool(results[0][1][1].any())


def test_rows_without_weight_and_nan():
    """Scores that are all -inf give 0 and add nothing; a NaN among a head's scores makes all of its group's NaN."""
    import paper_2608_13226_amd as cp
    a = _data([50, 60, 70], 4, 2, 64, 16, BF, "same")
    a["k_cache"].copy_(a["k_cache"].abs().nan_to_num(0.5))
    a["k_cache"][:, :, :, 0] = math.inf
    a["q"].copy_(a["q"].abs().clamp(min=0.01))
    a["q"][0, :, 0] = -1.0                                   # -inf everywhere
    a["q"][1, 0, 1] = math.nan                               # one head's scores NaN
    a["k_cache"][:, :, :, 0] = torch.where(torch.arange(a["k_cache"].shape[0], device="cuda")[:, None, None] >= 0, math.inf, 0.0)
    a["q"][1, 1:, 0], a["q"][2, :, 0] = -1.0, -1.0
    mass = torch.full((3, 2, 70), 0.25, device="cuda")
    v = a["v_cache"].nan_to_num(1.0)
    out, lse = cp.paged_attention_mass(a["q"], a["k_cache"], v, a["table"], a["lengths"], mass, max_length=70, return_lse=True)
    assert not bool(out[0].any()) and bool((lse[0] == -math.inf).all()) and bool((mass[0] == 0.25).all())
    assert bool(torch.isnan(out[1, 0]).all()) and bool(torch.isnan(mass[1, 0, :60]).all()) and bool((mass[1, 0, 60:] == 0.25).all())
    assert bool((mass[1, 1] == 0.25).all()) and not bool(out[1, 1:].any())


def test_a_nan_block_of_keys_or_values():
    """A key whose block is NaN makes the whole row NaN, a value that dims."""
    a = _data([40, 300], 4, 1, 128, 16, BF)
    page = a["table"][0, 0].long()
    a["v_scale"][page, 0, 3, 1] = 255
    out, lse = (x.cpu() for x in _check4(a))
    assert bool(torch.isnan(out[0, :, 32:64]).all()) and not bool(torch.isnan(out[0, :, :32]).any()) and not bool(torch.isnan(out[1]).any())
    a["k_scale"][a["table"][1, 2].long(), 0, 9, 0] = 255
    out, lse, mass = _check_mass(a)
    assert bool(torch.isnan(out[1]).all()) and bool(torch.isnan(mass[1]).all()) and not bool(torch.isnan(mass[0]).any())


def test_the_same_twice_and_shared_pages():
    """Equal bit for bit; sequences may share pages, each has masses of its own."""
    import paper_2608_13226_amd as cp
    a = _data([3000] * 3, 28, 4, 128, 64, BF)
    a["table"] = a["table"][:1].expand(3, -1).contiguous()
    a["lengths"] = torch.tensor([3000, 10, 2999], dtype=torch.int32, device="cuda")
    _check4(a)
    runs = []
    for _ in range(2):
        mass = torch.zeros(3, 4, 3000, device="cuda")
        runs.append([cp.paged_attention_mass(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], mass, k_scale=a["k_scale"],
                                             v_scale=a["v_scale"]), mass])
    assert all(torch.equal(x, y) for x, y in zip(*runs))
    _check_mass(a)


def test_masses_add_up_to_the_heads():
    a = _data([5000, 77], 28, 4, 128, 16, BF, "e4m3")
    import paper_2608_13226_amd as cp
    mass = torch.zeros(2, 4, 5000, device="cuda")
    for _ in range(3):
        cp.paged_attention_mass(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], mass, max_length=5000, k_scale=a["k_scale"],
                                v_scale=a["v_scale"])
    assert bool(((mass.double().sum(2) - 21).abs() < 21 * 2.0 ** -16).all())


def test_masses_without_alignment():
    """One sequence's part of an array of odd spans."""
    import paper_2608_13226_amd as cp
    for lengths in ([37], [3001]):
        a = _data(lengths, 8, 2, 64, 16, BF)
        pool = torch.zeros(3, 2, 3003, device="cuda").flatten()[1:]
        mass = pool[:2 * 3003].view(1, 2, 3003)
        _check_mass(a, span=3003, start=mass)
        assert not bool(pool[2 * 3003:].any())


def test_long_caches():
    """Slots past 2^31 bytes of codes and a sequence of 200000 tokens."""
    import paper_2608_13226_amd as cp
    g = torch.Generator(device="cuda").manual_seed(1)
    page, hk, d, n = 64, 4, 128, 200_001
    pages = (1 << 31) // (hk * page * d // 2) + 4000
    caches = [torch.randint(0, 256, (pages, hk, page, d // 2), device="cuda", generator=g, dtype=torch.uint8) for _ in range(2)]
    scales = [torch.randint(124, 128, (pages, hk, page, d // 32), device="cuda", generator=g, dtype=torch.uint8) for _ in range(2)]
    width = (n + page - 1) // page
    table = (pages - 1 - torch.randperm(width, device="cuda", generator=g)).to(torch.int32)[None]
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    q = (0.2 * torch.randn(1, 8, d, device="cuda", generator=g)).to(BF)
    mass = torch.zeros(1, hk, n, device="cuda")
    out = cp.paged_attention_mass(q, *caches, table, lengths, mass, k_scale=scales[0], v_scale=scales[1])
    at = torch.arange(n, device="cuda")
    slots = table[0].long()[at // page] * page + at % page
    k, v = (x.double() for x in cp.kv_gather(*caches, slots, BF, *scales))
    s = (k.transpose(0, 1).contiguous() @ q.double().view(hk, 2, d).transpose(1, 2).contiguous()) / math.sqrt(d)
    p = torch.softmax(s, 1)
    want = (p.transpose(1, 2).contiguous() @ v.transpose(0, 1).contiguous()).view(1, 8, d)
    a = dict(q=q, lengths=lengths)
    size = (p.transpose(1, 2).contiguous() @ v.transpose(0, 1).abs().contiguous()).view(1, 8, d)
    ref.assert_close(out, want.cpu(), BF, _work(a) * size.cpu(), "out")
    ref.assert_close(mass, p.sum(2)[None].cpu(), torch.float32, 2 * _work(a) * p.sum(2)[None].cpu(), "mass")
