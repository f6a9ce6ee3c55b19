"""coverprune_w4_matvec against its float64 statement."""
import pytest

from tests import serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


def _data(m, n, k, group, t, x8, zero, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + m + 31 * n + 7 * k)
    x = torch.randn(m, k, device="cuda", generator=g)
    xs = None
    if x8:
        xs = 0.01 + torch.rand(m, device="cuda", generator=g)
        x = (60.0 * x).clamp(-448, 448).to(E4M3)
    else:
        x = x.to(t)
    w = torch.randint(0, 256, (n, k // 2), device="cuda", generator=g, dtype=torch.uint8)
    s = (0.05 * torch.randn(n, k // group, device="cuda", generator=g)).to(t)
    z = torch.randint(0, 16, (n, k // group), device="cuda", generator=g, dtype=torch.uint8) if zero else None
    return x, w, s, z, xs


def _check(x, w, s, z, xs, out_dtype=None):
    import paper_2608_13226_amd as cp
    y = cp.w4_matvec(x, w, s, zero=z, x_scale=xs, out_dtype=out_dtype)
    want, work = ref.w4_matvec(x, w, s, z, xs)
    assert y.shape == want.shape and y.dtype == (out_dtype or s.dtype)
    ref.assert_close(y, want, y.dtype, work, f"m={x.shape[0]} n={w.shape[0]} k={x.shape[1]}")
    return y


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("t", [BF, F16])
@pytest.mark.parametrize("m,n,k,group", [
    (1, 1, 32, 32), (1, 16, 64, 32), (2, 33, 96, 96), (3, 15, 160, 32), (1, 128, 128, 128), (7, 48, 384, 128),
    (15, 17, 256, 256), (16, 100, 192, 64), (17, 64, 512, 128), (5, 1500, 1184, 32), (33, 130, 640, 64),
    (64, 257, 1024, 128), (65, 96, 320, 160), (130, 40, 896, 128), (1, 4608, 3584, 128), (4, 70, 4480, 4480),
    (9, 96, 2112, 96), (24, 300, 7168, 256),
    # many outputs: 64 a wave; and, with more than 16 rows, x shared in LDS
    (1, 16400, 256, 128), (6, 16390, 416, 32), (16, 4200, 576, 64), (17, 10250, 384, 128), (20, 10241, 160, 32),
    (33, 8200, 320, 32), (64, 8192, 1088, 64), (130, 8300, 2208, 96), (40, 8195, 2304, 32), (64, 8321, 256, 256)])
def test_products(m, n, k, group, t, x8):
    zero = (m + n) % 2 == 1
    print(f"w4 m={m} n={n} k={k} group={group} {t} x8={x8} zero={zero}", flush=True)
    data = _data(m, n, k, group, t, x8, zero)
    _check(*data)
    _check(*data, out_dtype=F32)


def test_every_code_and_place():
    """One row of x picks single codes out: every code value at every place of a 128-run."""
    import paper_2608_13226_amd as cp
    for t in (BF, F16):
        for group in (32, 128):
            k = n = 256
            codes = (torch.arange(n, device="cuda")[:, None] * 7 + torch.arange(k, device="cuda")) % 16
            w = (codes[:, 0::2] | codes[:, 1::2] << 4).to(torch.uint8)
            s = torch.ones(n, k // group, device="cuda", dtype=t)
            y = cp.w4_matvec(torch.eye(k, device="cuda", dtype=t), w, s, out_dtype=F32)
            assert torch.equal(y, (codes - 8).t().float()), (t, group)


def test_no_rows():
    import paper_2608_13226_amd as cp
    x, w, s, z, _ = _data(0, 32, 128, 128, BF, False, True)
    assert cp.w4_matvec(x, w, s, zero=z).shape == (0, 32)


@pytest.mark.parametrize("n", [100, 10300])
def test_rows_do_not_touch_each_other(n):
    """NaN or infinity in one row of x reaches that row's results only."""
    import paper_2608_13226_amd as cp
    x, w, s, z, _ = _data(20, n, 512, 128, BF, False, True)
    clean = cp.w4_matvec(x, w, s, zero=z)
    x[3, 7], x[18, 500] = float("nan"), float("inf")
    y = cp.w4_matvec(x, w, s, zero=z)
    keep = [i for i in range(20) if i not in (3, 18)]
    assert torch.equal(y[keep], clean[keep])
    assert not bool(torch.isfinite(y[3].float()).any())


def test_the_same_answer_every_time():
    import paper_2608_13226_amd as cp
    x, w, s, z, _ = _data(64, 1000, 3584, 128, BF, False, True)
    y = cp.w4_matvec(x, w, s, zero=z)
    for _ in range(5):
        assert torch.equal(cp.w4_matvec(x, w, s, zero=z), y)


def test_fed_by_the_norm():
    """The norm's 8-bit rows and scales are what the product takes."""
    import paper_2608_13226_amd as cp
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(6, 1024, device="cuda", generator=g).to(BF)
    gain = torch.ones(1024, device="cuda", dtype=BF)
    r = cp.rms_norm(x, gain, quantize=True)
    _, w, s, z, _ = _data(6, 200, 1024, 128, BF, False, True)
    _check(r.out, w, s, z, r.scale, out_dtype=F32)


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 6, 8, 9])
@pytest.mark.parametrize("n,k,group", [
    (31, 8224, 32), (20, 9216, 128), (17, 8256, 64), (50, 2048, 1024), (4130, 288, 32), (4100, 192, 64), (4113, 640, 128),
    (12300, 2048, 64)])
def test_few_rows(m, n, k, group, x8):
    """Rows that lanes share, a block's waves many and few, 16 to 64 outputs a wave."""
    print(f"w4 m={m} n={n} k={k} group={group} x8={x8}", flush=True)
    _check(*_data(m, n, k, group, BF if n % 2 else F16, x8, n % 3 != 0, seed=9))


@pytest.mark.parametrize("m", [2, 4, 7])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_few_rows_do_not_touch_each_other(m, group):
    import paper_2608_13226_amd as cp
    x, w, s, z, _ = _data(m, 200, 896, group, BF, False, True)
    clean = cp.w4_matvec(x, w, s, zero=z)
    x[1, 7] = float("nan")
    y = cp.w4_matvec(x, w, s, zero=z)
    keep = [i for i in range(m) if i != 1]
    assert torch.equal(y[keep], clean[keep])
    assert bool(torch.isnan(y[1].float()).all())


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("t", [BF, F16])
@pytest.mark.parametrize("m,n,k,group", [
    (17, 16390, 384, 128), (20, 16385, 160, 32), (33, 16400, 320, 32), (64, 16384, 1088, 64), (130, 16500, 1056, 96),
    (40, 16387, 2304, 32), (64, 16641, 256, 256), (32, 16400, 32, 32)])
def test_many_rows_and_outputs(m, n, k, group, t, x8):
    """x shared in LDS: one block of rows and several, turns and groups that end anywhere."""
    print(f"w4 m={m} n={n} k={k} group={group} {t} x8={x8}", flush=True)
    _check(*_data(m, n, k, group, t, x8, n % 2 == 1, seed=4))


def test_many_outputs_rows_do_not_touch_each_other():
    import paper_2608_13226_amd as cp
    x, w, s, z, _ = _data(20, 16500, 512, 128, BF, False, True)
    clean = cp.w4_matvec(x, w, s, zero=z)
    x[3, 7], x[18, 500] = float("nan"), float("inf")
    y = cp.w4_matvec(x, w, s, zero=z)
    keep = [i for i in range(20) if i not in (3, 18)]
    assert torch.equal(y[keep], clean[keep])
    assert not bool(torch.isfinite(y[3].float()).any())


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("m,n,k,group,t", [
    (17, 20490, 384, 128, BF), (20, 20481, 160, 32, F16), (32, 20500, 32, 32, BF), (33, 13701, 1088, 64, F16),
    (64, 10240, 2304, 32, BF), (64, 16384, 256, 256, F16), (64, 16385, 1056, 96, BF), (40, 22001, 320, 32, F16),
    (130, 8300, 416, 32, BF), (99, 6001, 2176, 128, BF), (300, 4100, 192, 64, F16)])
def test_rows_times_outputs(m, n, k, group, t, x8):
    """32 and 64 rows a block, up to a block a compute unit and past it, last blocks of few rows and outputs."""
    print(f"w4 m={m} n={n} k={k} group={group} {t} x8={x8}", flush=True)
    _check(*_data(m, n, k, group, t, x8, n % 2 == 1, seed=6))


@pytest.mark.parametrize("m,n", [(20, 20500), (64, 10300), (64, 17000)])
def test_rows_times_outputs_do_not_touch_each_other(m, n):
    import paper_2608_13226_amd as cp
    x, w, s, z, _ = _data(m, n, 512, 128, BF, False, True)
    clean = cp.w4_matvec(x, w, s, zero=z)
    x[3, 7], x[18, 500] = float("nan"), float("inf")
    y = cp.w4_matvec(x, w, s, zero=z)
    keep = [i for i in range(m) if i not in (3, 18)]
    assert torch.equal(y[keep], clean[keep])
    assert not bool(torch.isfinite(y[3].float()).any())


@pytest.mark.parametrize("t", [BF, F16])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("m,n,k,group", [(1, 40, 8320, 64), (3, 200, 896, 128), (7, 90, 320, 32), (20, 100, 512, 128), (40, 5000, 384, 96),
                                         (20, 20500, 512, 128), (64, 16700, 288, 32)])
def test_rows_with_infinities(m, n, k, group, zero, t):
    """An infinite x gives infinity of the sign of code - zero, NaN where that is 0 or two of them disagree; a sum of
    large x that float32 does not hold counts as the formula has it."""
    print(f"w4 infinities m={m} n={n} k={k} group={group} {t} zero={zero}", flush=True)
    x, w, s, z, _ = _data(m, n, k, group, t, False, zero, seed=11)
    inf = float("inf")
    x[0, 5] = inf
    if m > 1:
        x[m - 1, k - 1] = -inf
    if m > 2:
        x[1, 7], x[1, k // 2] = inf, -inf
    if m > 5:
        # Four large x of one sign at codes one above and one below the zero point.
        x[3, 0:4] = 1.5e38 if t == BF else 6e4
        at = torch.full((n,), 8, device="cuda", dtype=torch.uint8) if z is None else z[:, 0].clamp(1, 14)
        if z is not None:
            z[:, 0] = at
        w[:, 0] = (at + 1) | (at - 1) << 4
        w[:, 1] = (at - 1) | (at + 1) << 4
    for out_dtype in (None, F32):
        y = _check(x, w, s, z, None, out_dtype=out_dtype)
        assert bool(torch.isinf(y[0].float()).any()) and bool(torch.isnan(y[0].float()).any() == ((w[:, 2] >> 4) == (8 if z is None else z[:, 0])).any())
        if m > 5:
            assert bool(torch.isfinite(y[3].float()).all())
