"""How many bits of a weight reach the values that are attended to, and of a rotated key the codes it is held in."""
import math

import pytest

from tests import cache_ref, serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def _attend(a, mass, **kw):
    import paper_2608_13226_amd as cp
    scales = dict(k_scale=a["k_scale"], v_scale=a["v_scale"])
    args = a["q"], a["k_cache"], a["v_cache"]
    if mass:
        hk, span = a["k_cache"].shape[1], a["table"].shape[1] * a["k_cache"].shape[2]
        m = torch.zeros(a["q"].shape[0], hk, span, device="cuda")
        return cp.paged_attention_mass(*args, a["table"], a["lengths"], m, **scales, **kw)
    if a["k_cache"].dtype == torch.uint8:
        return cp.paged_attention4(*args, a["k_scale"], a["v_scale"], a["table"], a["lengths"], **kw)
    return cp.paged_attention(*args, a["table"], a["lengths"], **scales, **kw)


@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("held", ["same", "e4m3", "e2m1"])
@pytest.mark.parametrize("t", [BF, F16])
def test_weights_keep_float32s_bits(t, held, mass):
    """Two tokens whose values cancel and whose weights differ by 2^-14: what is left shows each weight's last bits.  (A third,
    without a value, has the largest weight, a power of two.)

    Relative to a weight: its exponent x, below 2.9, is rounded twice, and once more with 8 to 16 taken off it,
    ln 2 (2 * 2.9 * 2^-24 + 2^-21) = 1.2 * 2^-21; the exponential to a step, 2^-23; float16's two parts leave 2^-22, bfloat16's
    three 2^-25; six additions and two products of at most 1 add 8 * 2^-24 / 2.  Together below 2.5 * 2^-21."""
    g = torch.Generator(device="cuda").manual_seed(9)
    batch, heads, d, page = 64, 16, 64, 16
    k, v = (torch.zeros(1, 1, page, d, device="cuda") for _ in range(2))
    k[0, 0, :3, 0] = torch.tensor([1.0, 1.0, 1.5])
    k[0, 0, 1, 32] = 2.0 ** -6
    v[0, 0, 0], v[0, 0, 1] = 1.0, -1.0
    caches, scales = [], []
    for x in (k, v):
        codes, e = cache_ref.cut_cache(x, t) if held == "e2m1" else (x.to(E4M3 if held == "e4m3" else t), None)
        caches.append(codes)
        scales.append(e)
        if held == "e2m1":
            assert torch.equal(cache_ref.values(codes, e), ref.d64(x))
    q = torch.zeros(batch, heads, d, device="cuda")
    q[:, :, 0] = 0.5 + 1.5 * torch.rand(batch, heads, device="cuda", generator=g)
    q[:, :, 32] = 2.0 ** -8 * (1 + torch.rand(batch, heads, device="cuda", generator=g))
    q = q.to(t)
    a = dict(q=q, k_cache=caches[0], v_cache=caches[1], table=torch.zeros(batch, 1, dtype=torch.int32, device="cuda"),
             lengths=torch.full((batch,), 3, dtype=torch.int32, device="cuda"), k_scale=scales[0], v_scale=scales[1])
    out = _attend(a, mass, max_length=3, scale=1.0)
    x, more = ref.d64(q)[:, :, 0], ref.d64(q)[:, :, 32] * 2.0 ** -6
    p = [torch.exp(-x / 2), torch.exp(more - x / 2), torch.ones_like(x)]
    want, size = (y[..., None].expand(batch, heads, d) / sum(p)[..., None] for y in (p[0] - p[1], p[0] + p[1]))
    ref.assert_close(out, want, t, 2.5 * 2.0 ** -21 * size, "out")


@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("t,byte", [(F16, 141), (F16, 150), (F16, 254), (BF, 253), (BF, 254)])
@pytest.mark.parametrize("lengths,d,page", [([1, 40, 300], 128, 16), ([700, 65], 64, 64), ([3000], 96, 32)])
def test_values_past_the_queries_type_are_infinite(lengths, d, page, t, byte, mass):
    """A cache made from another type, or by another program: what the type does not hold is an infinity, which makes its
    dimension infinite (two of both signs: NaN) and no other."""
    g = torch.Generator(device="cuda").manual_seed(d + byte)
    batch, hq, hk = len(lengths), 4, 2
    width = (max(lengths) + page - 1) // page
    table = torch.randperm(batch * width, device="cuda", generator=g).view(batch, width).to(torch.int32)
    caches, scales = [], []
    for _ in range(2):
        codes, e = cache_ref.cut_cache(torch.randn(batch * width, hk, page, d, device="cuda", generator=g), t)
        caches.append(codes)
        scales.append(e)
    # The first and the last token's second block of each sequence.
    for b, n in enumerate(lengths):
        for j in (0, n - 1):
            scales[1][int(table[b, j // page]), :, j % page, 1] = byte
    q = torch.randn(batch, hq, d, device="cuda", generator=g).to(t)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    a = dict(q=q, k_cache=caches[0], v_cache=caches[1], table=table, lengths=n, k_scale=scales[0], v_scale=scales[1])
    out = _attend(a, mass, max_length=max(lengths))
    held = [cache_ref.values(c, e).to(t).cuda() for c, e in zip(caches, scales)]
    want, _, size = ref.attend(q, *held, table, n)
    assert bool(torch.isinf(want).any()) and bool(torch.isfinite(want[..., :32]).all())
    # As in the attention's own tests.
    size = torch.where(torch.isfinite(size), size, torch.zeros_like(size))
    ref.assert_close(out, want, t, 2.0 ** -24 * (60 * (d / 32 + 8) + max(lengths) / 32 + 100) * size, "out")


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("magnitude", [0.5, 0.5 * (1 + 2.0 ** -30), 0.5 * (1 - 2.0 ** -30), 0.5 * (1 + 2.0 ** -23), 0.5 * (1 + 2.0 ** -22)])
def test_a_key_next_to_the_lowest_border(magnitude, inter):
    """A quarter of the smallest power, 2^-127, is where code 0 ends, and below float32's normal numbers: a key just
    above it has code 1 (exact in float64: turned by nothing, times the magnitude)."""
    import paper_2608_13226_amd as cp
    k = torch.full((3, 2, 32), 2.0 ** -126, device="cuda").to(BF)
    k[1], k[2, 0, ::2] = -k[1], 0.0
    caches = [torch.zeros(3, 2, 1, w, dtype=torch.uint8, device="cuda") for w in (16, 16, 1, 1)]
    cp.kv_append4(None, k, k, torch.zeros(3, dtype=torch.int32, device="cuda"), torch.arange(3, device="cuda"),
                  torch.ones(16, device="cuda"), *caches, interleaved=inter, magnitude=magnitude)
    code, e = cache_ref.blocks(ref.d64(k) * magnitude, BF)
    assert torch.equal(caches[2][:, :, 0].cpu().int(), e) and bool((e == 2).all())
    got = cache_ref.unpack(caches[0][:, :, 0])
    # (-0 where nothing is left of a negative one, and a turned 0 may have either sign.)
    assert torch.equal(got & 7, code & 7) and torch.equal(got[code & 7 != 0], code[code & 7 != 0])
    assert bool((code & 7 != 0).any()) == (magnitude > 0.5)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("magnitude", [1.0, 1 + 2.0 ** -30, 1 - 2.0 ** -30])
def test_keys_at_borders_beside_the_largest(magnitude, inter):
    """Next to an element at the end of float32's range, whose block has the largest power, 2^125, elements just past a border
    of that power have the code beyond it."""
    import paper_2608_13226_amd as cp
    k = torch.full((2, 1, 32), 2.0 ** 123, device="cuda").to(BF)
    k[:, :, 1::4], k[:, :, 2::4] = 1.25 * 2.0 ** 125, -2.5 * 2.0 ** 125
    k[:, :, 4::8], k[:, :, 3::8] = 0.75 * 2.0 ** 125, torch.finfo(BF).max
    caches = [torch.zeros(2, 1, 1, w, dtype=torch.uint8, device="cuda") for w in (16, 16, 1, 1)]
    cp.kv_append4(None, k, k, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.arange(2, device="cuda"),
                  torch.ones(16, device="cuda"), *caches, interleaved=inter, magnitude=magnitude)
    code, e = cache_ref.blocks(ref.d64(k) * magnitude, BF)
    assert torch.equal(caches[2][:, :, 0].cpu().int(), e) and bool((e == 252).all())
    assert torch.equal(cache_ref.unpack(caches[0][:, :, 0]), code)
