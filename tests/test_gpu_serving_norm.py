"""coverprune_rms_norm against its float64 statement."""
import pytest

from tests import serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def _data(rows, d, t, residual, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * rows + d)
    x = torch.randn(rows, d, device="cuda", generator=g).to(t)
    w = (1.0 + 0.3 * torch.randn(d, device="cuda", generator=g)).to(t)
    r = (3.0 * torch.randn(rows, d, device="cuda", generator=g)).to(t) if residual else None
    return x, w, r


def _check(x, w, r, eps, got, quantize):
    d = x.shape[1]
    y, h = ref.rms_norm(x, w, eps, r)
    # The sum of squares in float32: lanes add up to 64 values each, then a tree.
    work = 2.0 ** -24 * (64 + 16) * y.abs()
    if r is not None:
        ref.assert_close(got.residual, h, x.dtype, 2.0 ** -24 * h.abs(), f"residual d={d}")
    else:
        assert got.residual is None
    if not quantize:
        assert got.scale is None
        ref.assert_close(got.out, y, x.dtype, work, f"norm d={d}")
        return
    scale = y.abs().amax(1) / 448.0
    ref.assert_close(got.scale, scale, F32, 2.0 ** -24 * 96 * scale, f"scale d={d}")
    s = got.scale.cpu().double()[:, None]
    ref.assert_e4m3(got.out, torch.where(s == 0, torch.zeros_like(y), y / s), f"codes d={d}")


@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("t", [BF, F16, F32])
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (1, 8), (5, 96), (300, 1000), (1, 3584), (33, 3584), (2, 4097),
                                    (2, 8192), (3, 20001), (2, 65536), (700, 129), (1030, 64), (2050, 512)])
def test_norm(rows, d, t, residual, quantize):
    import paper_2608_13226_amd as cp
    print(f"norm rows={rows} d={d} {t} residual={residual} quantize={quantize}", flush=True)
    x, w, r = _data(rows, d, t, residual)
    got = cp.rms_norm(x, w, eps=1e-5, residual=r, quantize=quantize)
    _check(x, w, r, 1e-5, got, quantize)


def test_rows_of_nothing_and_zeros():
    import paper_2608_13226_amd as cp
    x, w, r = _data(0, 3584, BF, True)
    got = cp.rms_norm(x, w, residual=r, quantize=True)
    assert got.out.shape == (0, 3584) and got.scale.shape == (0,)
    x, w, _ = _data(3, 520, BF, False)
    x[1] = 0
    got = cp.rms_norm(x, w, eps=1e-6, quantize=True)
    _check(x, w, None, 1e-6, got, True)
    assert float(got.scale[1]) == 0.0 and not d64_any(got.out[1])


def d64_any(t):
    return bool((ref.d64(t) != 0).any())


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_bad_row_stays_alone(bad):
    """An infinite or NaN element spoils its own row (as in the formula) and no other."""
    import paper_2608_13226_amd as cp
    x, w, _ = _data(9, 1000, BF, False)
    clean = cp.rms_norm(x, w, quantize=True)
    x[4, 333] = bad
    got = cp.rms_norm(x, w, quantize=True)
    keep = [i for i in range(9) if i != 4]
    assert torch.equal(got.scale[keep], clean.scale[keep])
    assert torch.equal(got.out.view(torch.uint8)[keep], clean.out.view(torch.uint8)[keep])
    assert bool(torch.isnan(got.scale[4]))
    y = cp.rms_norm(x, w).out.float()
    assert bool(torch.isnan(y[4, 333])) and bool(torch.isfinite(y[keep]).all())


def test_update_in_place_and_given_outputs():
    import paper_2608_13226_amd as cp
    x, w, r = _data(65, 3584, BF, True)
    want = cp.rms_norm(x, w, residual=r)
    mine = r.clone()
    out = torch.empty_like(x)
    got = cp.rms_norm(x, w, residual=mine, residual_out=mine, out=out)
    assert got.out.data_ptr() == out.data_ptr() and torch.equal(out, want.out) and torch.equal(mine, want.residual)


def test_large_values_do_not_overflow_the_output_scale():
    import paper_2608_13226_amd as cp
    x, w, _ = _data(4, 2048, F32, False)
    x = x * 1e15
    x[2] *= 1e-30
    got = cp.rms_norm(x, w, eps=0.0, quantize=True)
    _check(x, w, None, 0.0, got, True)


@pytest.mark.parametrize("xs,ws", [(1e-20, 1e-15), (1e17, 1e18), (1e-4, 1e-30), (1e10, 1e-25), (3e18, 1.0)])
def test_products_near_the_ends_of_float32(xs, ws):
    """Rows and weights whose products leave the range that the codes' one factor covers."""
    import paper_2608_13226_amd as cp
    x, w, _ = _data(5, 1024, F32, False)
    x, w = x * xs, w * ws
    x[3] = 0
    got = cp.rms_norm(x, w, eps=0.0 if xs < 1e10 else 1e-6, quantize=True)
    y, _ = ref.rms_norm(x, w, 0.0 if xs < 1e10 else 1e-6, None)
    y = torch.nan_to_num(y) if xs < 1e10 else y
    keep = [0, 1, 2, 4]
    # 0 / 0 in the formula: the zero row with eps = 0.
    assert xs >= 1e10 or bool(torch.isnan(got.scale[3]))
    scale = y.abs().amax(1) / 448.0
    ref.assert_close(got.scale[keep], scale[keep], F32, 2.0 ** -24 * 96 * scale[keep], "scale")
    ref.assert_e4m3(got.out.view(torch.uint8)[keep].view(got.out.dtype), (y / got.scale.cpu().double()[:, None])[keep], "codes")


@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("t", [BF, F16, F32])
@pytest.mark.parametrize("rows,d", [(9, 2), (5, 9), (17, 15), (40, 1001), (3, 8191), (4, 16385), (2, 40003), (2, 65535)])
def test_rows_that_begin_anywhere(rows, d, t, quantize):
    """d is no multiple of eight: no row but the first is aligned, every last run is short."""
    import paper_2608_13226_amd as cp
    print(f"norm rows={rows} d={d} {t} quantize={quantize}", flush=True)
    x, w, r = _data(rows, d, t, True, seed=4)
    # What lies around the outputs stays as it is.
    e = torch.float8_e4m3fn if quantize else t
    wide = torch.zeros(rows * d + 64, device="cuda", dtype=torch.uint8 if quantize else e)
    wide.view(torch.uint8).fill_(0x55)
    keep = torch.zeros(rows * d + 64, device="cuda", dtype=t)
    keep.view(torch.uint8).fill_(0x55)
    out = wide[:rows * d].view(e).view(rows, d)
    got = cp.rms_norm(x, w, eps=1e-5, residual=r, quantize=quantize, out=out, residual_out=keep[:rows * d].view(rows, d))
    _check(x, w, r, 1e-5, got, quantize)
    assert bool((wide[rows * d:].view(torch.uint8) == 0x55).all()) and bool((keep[rows * d:].view(torch.uint8) == 0x55).all())


@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("size,eps", [(1e-13, 1e-6), (1e-19, 1e20), (1e-22, 1e-6), (1e-22, 1.0), (1e-25, 1e-6), (1e-25, 1e-5),
                                      (1e-30, 1e-30), (1e-30, 1e-38), (1e-35, 1e-6), (1e-35, 1e-12), (1e-35, 1e-36)])
def test_rows_far_below_the_root_of_eps(size, eps, t, quantize):
    """eps alone under the root, or beside squares that float32 does not hold: small results, but not 0."""
    import paper_2608_13226_amd as cp
    x, w, r = _data(6, 1024, F32, True)
    x, w, r = (x * size).to(t), w.to(t), (r * size).to(t)
    # The kernel's eps is the nearest float32.
    eps = float(torch.tensor(eps, dtype=F32))
    _check(x, w, None, eps, cp.rms_norm(x, w, eps=eps, quantize=quantize), quantize)
    _check(x, w, r, eps, cp.rms_norm(x, w, eps=eps, residual=r, quantize=quantize), quantize)


@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("t", [BF, F32])
@pytest.mark.parametrize("size,eps", [(2e-39, 0.0), (3e-40, 0.0), (1e-40, 1e-45), (2e-39, 1e-38)])
@pytest.mark.parametrize("d", [8, 1000, 40003])
def test_subnormal_rows(d, size, eps, t, quantize):
    """Rows whose 1 / rms float32 does not hold: results of the usual size."""
    import paper_2608_13226_amd as cp
    x, w, _ = _data(5, d, F32, False)
    x, w = (x * size).to(t), w.to(t)
    assert bool((x != 0).any(1).all())
    eps = float(torch.tensor(eps, dtype=F32))
    _check(x, w, None, eps, cp.rms_norm(x, w, eps=eps, quantize=quantize), quantize)


@pytest.mark.parametrize("t", [BF, F16, F32])
@pytest.mark.parametrize("d", [200, 3584, 5001])
def test_codes_half_way_between_two(t, d):
    """Rows of n / 2 (n a whole number) times a row's factor, the largest 448 times it: half-way values go to the even code."""
    import paper_2608_13226_amd as cp
    g = torch.Generator(device="cuda").manual_seed(d)
    rows = 64
    # The factor's bits and the values' fill the type's.
    bits = {BF: 3, F16: 6, F32: 19}[t]
    m = 2.0 * torch.randint(0, 2 ** (bits - 1), (rows, 1), device="cuda", generator=g) + 1.0
    n = torch.randint(0, 32, (rows, d), device="cuda", generator=g).float()
    sign = 1.0 - 2.0 * torch.randint(0, 2, (rows, d), device="cuda", generator=g)
    want = n * 2.0 ** torch.randint(-3, 4, (rows, d), device="cuda", generator=g) * sign
    want[:, d // 3] = 448.0
    x = want * m * 2.0 ** -4
    assert torch.equal(x.to(t).float(), x)
    got = cp.rms_norm(x.to(t), torch.ones(d, device="cuda", dtype=t), quantize=True)
    assert torch.equal(got.out.float(), want.to(torch.float8_e4m3fn).float())
