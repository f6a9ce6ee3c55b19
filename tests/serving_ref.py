"""float64 statements of the serving operators, on the CPU, and the error
bounds that the GPU results are held to.  Plain loops and whole-array
arithmetic from the definitions; nothing is shared with the library."""
import math

import torch

HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
# Below the normal range of the type a rounding moves a value by up to this.
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}
E4M3 = torch.float8_e4m3fn


def d64(x):
    return None if x is None else x.detach().cpu().to(torch.float32).double() if x.dtype == E4M3 else x.detach().cpu().double()


def assert_close(got, want, dtype, slack, what):
    """|got - want| at most the rounding to dtype plus `slack` (a tensor or number, the bound on the float32 work)."""
    got, want = d64(got), want.double()
    slack = torch.as_tensor(slack, dtype=torch.float64).expand_as(want)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), f"{what}: infinities differ"
    got, want, slack = got[fine], want[fine], slack[fine]
    room = (want.abs() + slack) * HALF_ULP[dtype] + TINY[dtype] + slack
    over = (got - want).abs() - room
    if over.numel():
        i = int(over.argmax())
        assert float(over[i]) <= 0, f"{what}: {float(got[i])} for {float(want[i])}, over the bound {float(room[i]):.3g} by {float(over[i]):.3g}"


def assert_e4m3(codes, want, what, rel=2.0 ** -18):
    """codes (float8) within rounding of `want`: half a step of 3 bits after
    the leading one, or of the smallest exponent, and float32 work of `rel`."""
    codes, want = d64(codes), want.double()
    assert torch.equal(torch.isnan(codes), torch.isnan(want)), f"{what}: NaN in other places"
    ok = ~torch.isnan(want)
    codes, want = codes[ok], want[ok].clamp(-448.0, 448.0)
    room = torch.maximum(want.abs() * 2.0 ** -4, torch.tensor(2.0 ** -10, dtype=torch.float64)) + rel * want.abs()
    assert bool(((codes - want).abs() <= room).all()), f"{what}: a code is more than half a step off"


def rms_norm(x, w, eps, residual=None):
    h = d64(x) if residual is None else d64(x) + d64(residual)
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * d64(w)
    return y, h


def unpack_w4(weight, scale, zero):
    """[n, k] float64 weights, and their largest summands |code| + |zero| times |scale|."""
    w = weight.cpu()
    n, half = w.shape
    codes = torch.empty(n, 2 * half, dtype=torch.float64)
    codes[:, 0::2] = (w & 15).double()
    codes[:, 1::2] = (w >> 4).double()
    group = 2 * half // scale.shape[1]
    s = d64(scale).repeat_interleave(group, 1)
    z = (torch.full_like(d64(scale), 8.0) if zero is None else d64(zero)).repeat_interleave(group, 1)
    return (codes - z) * s, (codes + z) * s.abs()


def w4_matvec(x, weight, scale, zero=None, x_scale=None):
    w, big = unpack_w4(weight, scale, zero)
    x = d64(x)
    if x_scale is not None:
        x = x * d64(x_scale)[:, None]
    k = x.shape[1]
    # Sums of 32 products at a time, one after another, then a few more steps.
    return x @ w.t(), (k / 32 + 48) * 2.0 ** -23 * (x.abs() @ big.t())


def rotate(x, positions, inv_freq, interleaved, magnitude):
    """[tokens, heads, d] rotated, and |a| + |b| of each element's pair."""
    x = d64(x).clone()
    size = torch.zeros_like(x)
    if inv_freq is None:
        return x, size
    half = inv_freq.shape[0]
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = positions.cpu().double() * float(inv_freq[i].double())
        c, s = magnitude * torch.cos(angle)[:, None], magnitude * torch.sin(angle)[:, None]
        xa, xb = x[:, :, a].clone(), x[:, :, b].clone()
        x[:, :, a], x[:, :, b] = xa * c - xb * s, xb * c + xa * s
        size[:, :, a] = size[:, :, b] = (xa.abs() + xb.abs()) * abs(magnitude)
    return x, size


def attend(q, k_cache, v_cache, table, lengths, window=0, scale=None, k_scale=None, v_scale=None):
    """out, lse and the sum of p |v| that bounds out's float32 work."""
    batch, hq, d = q.shape
    hk, page = k_cache.shape[1], k_cache.shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = torch.zeros(batch, hq, d, dtype=torch.float64)
    size = torch.zeros(batch, hq, d, dtype=torch.float64)
    lse = torch.full((batch, hq), -math.inf, dtype=torch.float64)
    qd = d64(q)
    for b in range(batch):
        n = int(lengths[b])
        lo = max(0, n - window) if window else 0
        if n <= lo:
            continue
        at = torch.arange(lo, n)
        pages = table[b].cpu().long()[at // page].to(k_cache.device)
        off = (at % page).to(k_cache.device)
        for h in range(hq):
            kh = h // (hq // hk)
            k, v = d64(_rows(k_cache, pages, kh, off)), d64(_rows(v_cache, pages, kh, off))
            if k_scale is not None:
                k = k * float(k_scale[kh])
            if v_scale is not None:
                v = v * float(v_scale[kh])
            s = (k * qd[b, h]).sum(1) * scale
            p = torch.softmax(s, 0)
            out[b, h] = (p[:, None] * v).sum(0)
            size[b, h] = (p[:, None] * v.abs()).sum(0)
            lse[b, h] = torch.logsumexp(s, 0)
    return out, lse, size


def _rows(cache, pages, head, off):
    if cache.dtype == E4M3:
        return cache.view(torch.uint8)[pages, head, off].view(E4M3)
    return cache[pages, head, off]
