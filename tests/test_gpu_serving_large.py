"""The serving operators where one launch of HIP, less than 2^32 work items a
dimension, does not hold the grid: the answers are those of the same rows in
smaller calls."""
import pytest

from tests import serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16 = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    free, _ = torch.cuda.mem_get_info()
    if free < 80 << 30:
        pytest.skip("not enough free memory on this card")
    yield
    torch.cuda.empty_cache()


def _repeated(base, rows):
    """base's rows over and over, `rows` in all."""
    n = base.shape[0]
    out = torch.empty(rows, *base.shape[1:], device="cuda", dtype=base.dtype)
    whole = rows // n * n
    out[:whole].view(-1, *base.shape).copy_(base)
    out[whole:] = base[:rows - whole]
    return out


def _same(big, base):
    """big is base's rows over and over."""
    n = base.shape[0]
    whole = big.shape[0] // n * n
    parts = big[:whole].view(-1, *base.shape)
    for i in range(0, parts.shape[0], 1 << 12):
        part = parts[i:i + (1 << 12)]
        if not bool((part == base).all()):
            return False
    return torch.equal(big[whole:], base[:big.shape[0] - whole])


@pytest.mark.parametrize("quantize", [False, True])
def test_norm(quantize):
    """More rows than blocks of a wave in one launch."""
    import paper_2608_13226_amd as cp
    rows, d = 2 ** 26 + 5, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    base = torch.randn(1 << 14, d, device="cuda", generator=g).to(BF)
    w = torch.randn(d, device="cuda", generator=g).to(BF)
    want = cp.rms_norm(base, w, residual=base, quantize=quantize)
    x = _repeated(base, rows)
    got = cp.rms_norm(x, w, residual=x, quantize=quantize)
    assert _same(got.out.view(torch.uint8), want.out.view(torch.uint8)) and _same(got.residual, want.residual)
    assert not quantize or _same(got.scale[:, None], want.scale[:, None])


def test_append():
    import paper_2608_13226_amd as cp
    tokens, page = 2 ** 27 + 9, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    k = torch.randn(tokens, 1, 1, device="cuda", generator=g).to(F16)
    v = torch.randn(tokens, 1, 1, device="cuda", generator=g).to(F16)
    pages = (tokens + page - 1) // page
    k_cache, v_cache = (torch.zeros(pages, 1, page, 1, device="cuda", dtype=F16) for _ in range(2))
    slots = torch.arange(tokens - 1, -1, -1, device="cuda")
    cp.kv_append(None, k, v, torch.zeros(tokens, dtype=torch.int32, device="cuda"), slots, None, k_cache, v_cache)
    for x, cache in ((k, k_cache), (v, v_cache)):
        assert torch.equal(cache.view(-1)[:tokens], x.view(-1).flip(0)) and not bool(cache.view(-1)[tokens:].any())


@pytest.mark.parametrize("m,n", [(1, 2 ** 30 + 40), (17, 2 ** 29 + 200)])
def test_products(m, n):
    """Few rows, and many, over more outputs than one launch has blocks for."""
    import paper_2608_13226_amd as cp
    k = 32
    g = torch.Generator(device="cuda").manual_seed(m)
    # As many outputs as take the same kernel.
    some = 1 << 17 if m > 1 else 1 << 14
    x = torch.randn(m, k, device="cuda", generator=g).to(BF)
    w = torch.randint(0, 256, (some, k // 2), device="cuda", generator=g, dtype=torch.uint8)
    s = torch.rand(some, 1, device="cuda", generator=g).to(BF)
    want = cp.w4_matvec(x, w, s)
    y = cp.w4_matvec(x, _repeated(w, n), _repeated(s, n))
    for i in range(m):
        assert _same(y[i, :, None], want[i, :, None]), f"row {i}"


def test_as_many_rows_of_x_as_allowed():
    import paper_2608_13226_amd as cp
    m, n, k = 2 ** 20, 16, 32
    g = torch.Generator(device="cuda").manual_seed(4)
    base = torch.randn(1 << 14, k, device="cuda", generator=g).to(BF)
    w = torch.randint(0, 256, (n, k // 2), device="cuda", generator=g, dtype=torch.uint8)
    s = torch.rand(n, 1, device="cuda", generator=g).to(BF)
    y = cp.w4_matvec(_repeated(base, m), w, s)
    want, work = ref.w4_matvec(base, w, s)
    ref.assert_close(y[:1 << 14], want, BF, work, "first rows")
    assert _same(y, y[:1 << 14])
