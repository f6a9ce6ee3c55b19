"""coverprune_kv_append against its float64 statement."""
import pytest

from tests import serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


def _qkv(tokens, hq, hk, d, t, g, pad=0):
    """Views of one projection's output; `pad` more elements a row move the rows off 16 bytes."""
    wide = torch.randn(tokens, (hq + 2 * hk) * d + pad, device="cuda", generator=g).to(t)[:, pad:]
    return (wide[:, :hq * d].view(tokens, hq, d) if not pad else wide[:, :hq * d].unflatten(1, (hq, d)),
            wide[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d)), wide[:, (hq + hk) * d:].unflatten(1, (hk, d)))


def _run(tokens, hq, hk, d, rot, page, t, c, interleaved, pad=0, magnitude=1.0, span=5000, drop=False, with_q=True):
    import paper_2608_13226_amd as cp
    g = torch.Generator(device="cuda").manual_seed(tokens + 3 * d + rot + page)
    q, k, v = _qkv(tokens, hq, hk, d, t, g, pad)
    positions = torch.randint(0, span, (tokens,), device="cuda", generator=g, dtype=torch.int32)
    inv = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda") / max(rot, 1)) if rot else None
    pages = (tokens + page - 1) // page + 3
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:tokens]
    if drop:
        slots[::3] = -1 - torch.arange(len(slots[::3]), device="cuda")
        slots[1::7] = pages * page + torch.arange(len(slots[1::7]), device="cuda")
    # What no token goes to has to stay as it is, NaN included.
    bits = torch.uint8 if c == E4M3 else torch.int16
    caches = [torch.randint(0, 100, (pages, hk, page, d), device="cuda", generator=g).to(bits).view(c) for _ in range(2)]
    for x in caches:
        x.view(bits)[:, :, 0, 0] = 0x7f if c == E4M3 else 0x7fff
    before = [x.view(bits).clone() for x in caches]
    eight = c == E4M3
    ks = 0.005 + 0.01 * torch.rand(hk, device="cuda", generator=g) if eight else None
    vs = 0.005 + 0.01 * torch.rand(hk, device="cuda", generator=g) if eight else None
    got = cp.kv_append(q if with_q else None, k, v, positions, slots, inv, caches[0], caches[1], interleaved=interleaved,
                       magnitude=magnitude, k_scale=ks, v_scale=vs)

    # The angle is within 2^-23 of a turn, and sine and cosine within 2 ulp: 2^-20 of the pair's size in all.
    if with_q:
        want, size = ref.rotate(q, positions, inv, interleaved, magnitude)
        ref.assert_close(got, want, t, 2.0 ** -20 * size, "q")
    else:
        assert got is None
    kept = (slots >= 0) & (slots < pages * page)
    pg, off = slots[kept] // page, slots[kept] % page
    k64, ksize = ref.rotate(k, positions, inv, interleaved, magnitude)
    for name, cache, was, want, size, scale in (("k", caches[0], before[0], k64, ksize, ks),
                                                ("v", caches[1], before[1], ref.d64(v), 0 * ksize, vs)):
        rows = ref._rows(cache.transpose(1, 2), pg, off, slice(None))
        w, sz = want[kept.cpu()], size[kept.cpu()]
        if eight:
            den = ref.d64(scale)[:, None]
            codes, near = ref.d64(rows), (w / den).clamp(-448, 448)
            step = torch.maximum(near.abs() * 2.0 ** -4, torch.tensor(2.0 ** -10, dtype=torch.float64))
            assert bool(((codes - near).abs() <= step + 2.0 ** -18 * (near.abs() + sz / den)).all()), name
        else:
            ref.assert_close(rows, w, t, 2.0 ** -20 * sz, name)
        after = cache.view(bits).clone()
        touched = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
        touched[pg, off] = True
        same = ~touched[:, None, :, None].expand_as(after)
        assert torch.equal(after[same], was[same]), f"{name}: a slot without a token changed"


@pytest.mark.parametrize("c8", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,hq,hk,d,rot,page,t", [
    (1, 28, 4, 128, 128, 16, BF), (3, 4, 4, 64, 32, 1, F16), (37, 8, 1, 256, 256, 7, BF), (5, 6, 2, 96, 96, 50, F16),
    (130, 16, 2, 128, 64, 64, BF), (9, 3, 3, 80, 20, 16, BF), (2, 2, 1, 10, 6, 3, F16), (4, 1, 1, 7, 2, 5, BF),
    (11, 4, 2, 192, 0, 16, BF), (6, 5, 5, 72, 72, 32, BF),
    # runs of four; many heads of few tokens, spread over blocks
    (21, 8, 2, 96, 24, 16, F16), (7, 3, 1, 36, 8, 4, BF), (1, 112, 16, 96, 48, 100, BF), (600, 3, 1, 64, 64, 16, F16),
    (1025, 2, 1, 128, 128, 64, BF)])
def test_append(tokens, hq, hk, d, rot, page, t, interleaved, c8):
    print(f"append tokens={tokens} heads={hq}/{hk} d={d} rot={rot} page={page} {t} inter={interleaved} c8={c8}", flush=True)
    _run(tokens, hq, hk, d, rot, page, t, E4M3 if c8 else t, interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pad", [1, 4])
def test_rows_off_16_bytes(pad, interleaved):
    _run(17, 8, 2, 128, 128, 16, BF, BF, interleaved, pad=pad)


def test_tokens_without_a_slot():
    _run(100, 8, 2, 64, 64, 16, BF, BF, False, drop=True)
    _run(100, 8, 2, 64, 64, 16, BF, E4M3, True, drop=True)


@pytest.mark.parametrize("span", [200000, 2 ** 31 - 1])
def test_far_positions(span):
    _run(40, 4, 2, 128, 128, 16, BF, BF, False, span=span, magnitude=1.3)
    _run(40, 4, 2, 128, 128, 16, F16, F16, True, span=span)


def test_without_queries_and_without_tokens():
    import paper_2608_13226_amd as cp
    _run(12, 4, 2, 128, 128, 16, BF, BF, False, with_q=False)
    q = torch.empty(0, 4, 128, device="cuda", dtype=BF)
    k = torch.empty(0, 2, 128, device="cuda", dtype=BF)
    cache = torch.zeros(3, 2, 16, 128, device="cuda", dtype=BF)
    out = cp.kv_append(q, k, k, torch.empty(0, dtype=torch.int32, device="cuda"),
                       torch.empty(0, dtype=torch.int64, device="cuda"), torch.ones(64, device="cuda"), cache, cache.clone())
    assert out.shape == (0, 4, 128)


@pytest.mark.parametrize("interleaved", [False, True])
def test_queries_in_place(interleaved):
    import paper_2608_13226_amd as cp
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn(33, 28, 128, device="cuda", generator=g).to(BF)
    k = torch.randn(33, 4, 128, device="cuda", generator=g).to(BF)
    pos = torch.arange(33, device="cuda", dtype=torch.int32) * 11
    slots = torch.arange(33, device="cuda")
    inv = 10000.0 ** (-torch.arange(0, 96, 2, device="cuda") / 96)
    caches = [torch.zeros(3, 4, 16, 128, device="cuda", dtype=BF) for _ in range(2)]
    want = cp.kv_append(q, k, k, pos, slots, inv, *caches, interleaved=interleaved)
    cp.kv_append(q, k, k, pos, slots, inv, *caches, interleaved=interleaved, q_out=q)
    assert torch.equal(q, want)


def test_a_cache_past_32_bits():
    """Slots whose byte offset does not fit 32 bits."""
    import paper_2608_13226_amd as cp
    pages, hk, page, d = 70000, 4, 64, 128                      # 4.3 GiB a cache
    k_cache = torch.empty(pages, hk, page, d, device="cuda", dtype=BF)
    v_cache = torch.empty(pages, hk, page, d, device="cuda", dtype=BF)
    g = torch.Generator(device="cuda").manual_seed(3)
    k = torch.randn(4, hk, d, device="cuda", generator=g).to(BF)
    v = torch.randn(4, hk, d, device="cuda", generator=g).to(BF)
    slots = torch.tensor([0, pages * page - 1, 69999 * page, 35000 * page + 5], device="cuda")
    cp.kv_append(None, k, v, torch.zeros(4, dtype=torch.int32, device="cuda"), slots, None, k_cache, v_cache)
    for i, s in enumerate(slots.tolist()):
        assert torch.equal(k_cache[s // page, :, s % page], k[i]) and torch.equal(v_cache[s // page, :, s % page], v[i])


@pytest.mark.parametrize("c8", [False, True])
@pytest.mark.parametrize("tokens,hq,hk,d,rot,page,interleaved,pad", [
    (2051, 1, 1, 64, 64, 7, False, 0), (2053, 2, 2, 64, 16, 16, True, 0), (1031, 4, 1, 128, 64, 50, False, 0),
    (2500, 3, 1, 96, 96, 128, False, 0), (2049, 2, 1, 36, 8, 16, True, 4), (4099, 1, 1, 7, 2, 5, False, 0),
    (2061, 1, 1, 256, 256, 1, False, 1), (1030, 16, 4, 64, 32, 64, True, 0)])
def test_many_tokens_of_few_heads(tokens, hq, hk, d, rot, page, interleaved, pad, c8):
    """Blocks of several tokens, the last of them short, some tokens without a slot."""
    print(f"append tokens={tokens} heads={hq}/{hk} d={d} rot={rot} page={page} c8={c8}", flush=True)
    _run(tokens, hq, hk, d, rot, page, BF, E4M3 if c8 else BF, interleaved, pad=pad, drop=True)
