"""coverprune_kv_evict against its statement: who stays, where, with rows, exponents and masses."""
import math

import pytest

from tests import cache_ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def _data(lengths, hk, d, page, held, seed=0, ties=False):
    g = torch.Generator(device="cuda").manual_seed(seed + len(lengths) + d + page)
    b = len(lengths)
    width = max(1, (max(lengths) + page - 1) // page)
    pages = b * width + 2
    wide = {"e2m1": d // 2, "e4m3": d}.get(held, d)

    def bits(w, t):
        x = torch.randint(0, 256, (pages, hk, page, w * (2 if t in (BF, F16) else 1)), device="cuda", generator=g, dtype=torch.uint8)
        return x.view(t)

    t = {"e2m1": torch.uint8, "e4m3": E4M3, "bf16": BF, "f16": F16}[held]
    k, v = bits(wide, t), bits(wide, t)
    ks, vs = (bits(d // 32, torch.uint8), bits(d // 32, torch.uint8)) if held == "e2m1" else (None, None)
    table = torch.randperm(pages, device="cuda", generator=g)[:b * width].view(b, width).to(torch.int32)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    span = max(1, max(lengths)) + 3
    mass = torch.randint(0, 5, (b, hk, span), device="cuda", generator=g).float() if ties else torch.exp(3 * torch.randn(b, hk, span, device="cuda", generator=g))
    return dict(k_cache=k, v_cache=v, table=table, lengths=n, mass=mass, k_scale=ks, v_scale=vs)


def _raw(x):
    return x.view(torch.uint8).cpu()


def _check(a, keep, recent=0, sink=0, in_place=False, **kw):
    import paper_2608_13226_amd as cp
    kw.setdefault("max_length", max(1, int(a["lengths"].max())))
    names = [x for x in ("k_cache", "v_cache", "k_scale", "v_scale") if a[x] is not None]
    before = {x: _raw(a[x]).clone() for x in names}
    mass = a["mass"].cpu()
    r = cp.kv_evict(**a, keep=keep, recent=recent, sink=sink, mass_out=a["mass"] if in_place else None, **kw)
    b, hk, span = mass.shape
    page = a["k_cache"].shape[2]
    lengths, table = a["lengths"].cpu().tolist(), a["table"].cpu().long()
    kept = torch.full((b, hk, keep), -1, dtype=torch.int32)
    left = torch.zeros(b, hk, span)
    want = {x: before[x].clone() for x in names}
    for i in range(b):
        n = min(max(lengths[i], 0), kw["max_length"])
        for h in range(hk):
            places = torch.tensor(cache_ref.evict(mass[i, h].tolist(), n, keep, recent, sink), dtype=torch.long)
            m = len(places)
            kept[i, h, :m] = places.int()
            left[i, h, :m] = mass[i, h][places]
            j = torch.arange(m)
            for x in names:
                want[x][table[i][j // page], h, j % page] = before[x][table[i][places // page], h, places % page]
    assert torch.equal(r.kept.cpu(), kept), "kept"
    assert torch.equal(r.lengths.cpu(), torch.tensor([min(max(n, 0), kw["max_length"], keep) for n in lengths], dtype=torch.int32))
    assert torch.equal(r.mass.cpu().nan_to_num(nan=-7.0), left.nan_to_num(nan=-7.0)), "mass"
    for x in names:
        assert torch.equal(_raw(a[x]), want[x]), x
    return r


@pytest.mark.parametrize("held", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("lengths,hk,d,page,keep,recent,sink", [
    ([1], 1, 64, 16, 1, 0, 0), ([2], 1, 64, 16, 1, 0, 0), ([2], 2, 64, 16, 1, 1, 0), ([2], 1, 32, 1, 1, 0, 1),
    ([0, 1, 5, 6, 7, 100], 4, 128, 16, 6, 2, 1), ([1000, 999, 3], 2, 96, 50, 900, 128, 4), ([1000, 999, 3], 2, 96, 50, 100, 100, 0),
    ([1025, 2048, 2049], 1, 64, 64, 1024, 0, 0), ([4097], 3, 128, 7, 4096, 4000, 96), ([5000, 20, 4999], 2, 256, 100, 17, 5, 12),
    ([3333, 3000], 4, 192, 128, 2999, 0, 7), ([700] * 9, 2, 64, 32, 636, 300, 0), ([20000, 17], 1, 128, 64, 2000, 32, 4),
    ([64, 65], 1, 64, 16, 5000, 64, 1)])
def test_evict(lengths, hk, d, page, keep, recent, sink, held):
    print(f"evict {lengths} hk={hk} d={d} page={page} keep={keep} recent={recent} sink={sink} {held}", flush=True)
    _check(_data(lengths, hk, d, page, held), keep, recent, sink)


@pytest.mark.parametrize("keep,recent,sink", [(500, 0, 0), (500, 100, 3), (1, 0, 0), (900, 900, 0), (900, 10, 890), (999, 0, 0)])
def test_ties_go_to_the_earlier(keep, recent, sink):
    _check(_data([1000, 1000, 950], 2, 64, 16, "bf16", ties=True), keep, recent, sink)
    a = _data([1000], 2, 64, 16, "e2m1")
    a["mass"].zero_()
    _check(a, keep, recent, sink)


def test_masses_of_every_kind():
    """Infinities, NaN of either sign, zeros of either sign, negative and subnormal ones."""
    a = _data([600, 601, 602], 2, 64, 16, "f16", ties=True)
    odd = torch.tensor([math.inf, -math.inf, math.nan, -math.nan, 0.0, -0.0, -1.0, 1e-42, -1e-42, 3e38, 1.0, 2.0], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    a["mass"].copy_(odd[torch.randint(0, len(odd), a["mass"].shape, device="cuda", generator=g)])
    for keep, recent, sink in ((550, 10, 2), (300, 0, 0), (100, 50, 50), (2, 1, 0)):
        _check({x: y.clone() if y is not None else None for x, y in a.items()}, keep, recent, sink)


def test_in_place_masses_and_an_eviction_after_another():
    a = _data([3000, 2500], 2, 128, 64, "e2m1")
    r = _check(a, 2600, 64, 4, in_place=True)
    assert r.mass.data_ptr() == a["mass"].data_ptr()
    a["lengths"] = r.lengths
    r = _check(a, 1000, 64, 4, in_place=True, max_length=2600)
    a["lengths"] = r.lengths
    _check(a, 1000, 64, 4, in_place=True, max_length=1000)


def test_max_length_cuts_and_lengths_below_zero():
    a = _data([500, 400, 300], 1, 64, 16, "bf16")
    a["lengths"] = torch.tensor([500, -4, 300], dtype=torch.int32, device="cuda")
    _check(a, 350, 5, 1, max_length=400)
    import paper_2608_13226_amd as cp
    b, c = _data([500, 400], 1, 64, 16, "bf16"), _data([500, 400], 1, 64, 16, "bf16")
    x = cp.kv_evict(**b, keep=100)
    y = cp.kv_evict(**c, keep=100, max_length=500)
    assert all(torch.equal(p, q) for p, q in zip(x, y)) and torch.equal(_raw(b["k_cache"]), _raw(c["k_cache"]))


@pytest.mark.parametrize("held,d", [("e4m3", 8), ("e4m3", 24), ("bf16", 8), ("f16", 1000), ("e2m1", 32), ("e2m1", 4096), ("bf16", 4096)])
def test_rows_of_any_width(held, d):
    _check(_data([200, 150], 2, d, 16, held), 100, 30, 2)


@pytest.mark.parametrize("n,keep,recent", [(131072, 65536, 1024), (131072, 131008, 128), (70001, 7, 3), (300000, 200000, 0)])
def test_long_sequences(n, keep, recent):
    print(f"evict {n} keep {keep} recent {recent}", flush=True)
    _check(_data([n], 1, 64, 64, "e2m1"), keep, recent, 4)
    _check(_data([n], 1, 64, 64, "e2m1", ties=True), keep, recent, 0)


def test_many_sequences_and_heads():
    _check(_data([3 + i % 40 for i in range(200)], 16, 64, 16, "e2m1", ties=True), 20, 4, 2)


def test_pages_outside_the_cache_are_clamped():
    """As in attention: an entry past the cache counts as the last page."""
    a = _data([40], 1, 64, 16, "bf16")
    last = a["k_cache"].shape[0] - 1
    a["table"][0] = torch.tensor([0, 1, last], dtype=torch.int32)
    b = {x: y.clone() if y is not None else None for x, y in a.items()}
    b["table"][0, 2] = 2 ** 31 - 1
    import paper_2608_13226_amd as cp
    x, y = cp.kv_evict(**a, keep=20, recent=4), cp.kv_evict(**b, keep=20, recent=4)
    assert torch.equal(x.kept, y.kept) and torch.equal(_raw(a["v_cache"]), _raw(b["v_cache"]))


@pytest.mark.parametrize("lengths,hk,keep,recent,sink,ties", [
    ([20000, 16384, 2500, 16000], 2, 2500, 100, 5, False), ([40000, 39000], 2, 20000, 15000, 64, True),
    ([16385], 1, 4000, 0, 0, True), ([30000, 12], 1, 29000, 29000, 0, False), ([30000], 2, 5000, 4000, 1000, False),
    ([16384, 16383], 2, 16000, 128, 4, True), ([16384], 1, 16383, 0, 0, False), ([16385, 9], 1, 16384, 1, 0, True),
    ([300000, 299999], 1, 150000, 100, 10, True), ([5000] * 4, 3, 2400, 300, 0, False), ([16384] * 2, 1, 8000, 8000, 0, False)])
def test_many_rows(lengths, hk, keep, recent, sink, ties):
    """Those that go in several launches, or nearly: chunks, boundaries inside them, sequences that are short enough beside them."""
    for held in ("e2m1", "bf16"):
        a = _data(lengths, hk, 64, 50, held, ties=ties)
        _check({x: y.clone() if y is not None else None for x, y in a.items()}, keep, recent, sink)
        a["mass"][:, 0, ::7] = math.nan
        a["mass"][:, 0, 3::11] = -math.inf
        _check(a, keep, recent, sink, in_place=True)


def test_all_masses_equal_in_a_long_sequence():
    a = _data([50000], 2, 32, 64, "e2m1")
    a["mass"].zero_()
    _check(a, 20000, 64, 4)


@pytest.mark.parametrize("n,keep", [(3000, 2900), (9000, 5000), (30000, 20000)])
def test_masses_without_alignment(n, keep):
    a = _data([n], 2, 64, 16, "bf16")
    x = a["mass"]
    a["mass"] = torch.empty(x.numel() + 1, device="cuda")[1:].view(x.shape)
    a["mass"].copy_(x)
    _check(a, keep, 10, 2, in_place=True)


def test_exponents_without_alignment():
    a = _data([3000, 700], 2, 128, 16, "e2m1")
    for name in ("k_scale", "v_scale"):
        x = a[name]
        y = torch.empty(x.numel() + 1, dtype=torch.uint8, device="cuda")[1:].view(x.shape)
        y.copy_(x)
        a[name] = y
    _check(a, 500, 50, 2)
