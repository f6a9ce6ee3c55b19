"""float64 statements of the operators that keep a session's cache small, on the
CPU: 4-bit blocks, reading them, masses, eviction.  Plain loops from the
definitions; nothing is shared with the library."""
import math

import torch

from tests import serving_ref as ref

E4M3 = torch.float8_e4m3fn
LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
POWERS = {torch.bfloat16: (-125, 125), torch.float16: (-23, 13)}


def blocks(x, dtype):
    """Rows x [..., d] (float64) cut into blocks of 32: codes [..., d] of 0 to 15, exponent bytes [..., d / 32]."""
    low, high = POWERS[dtype]
    b = x.unflatten(-1, (-1, 32))
    bad = ~torch.isfinite(b).all(-1)
    b = torch.where(bad[..., None], torch.zeros_like(b), b)
    top = b.abs().amax(-1)
    e = torch.full(top.shape, low, dtype=torch.int32)
    for i in range(low, high):
        e = torch.where(top > 6.0 * 2.0 ** i, torch.full_like(e, i + 1), e)
    y = b.abs() / torch.pow(2.0, e.double())[..., None]
    code = torch.zeros(y.shape, dtype=torch.uint8)
    for i in range(7):
        middle = (LEVELS[i] + LEVELS[i + 1]) / 2
        # A tie goes to the even code: up from odd ones only.
        code += (y >= middle if i % 2 else y > middle).to(torch.uint8)
    code += 8 * torch.signbit(b).to(torch.uint8)
    return torch.where(bad[..., None], torch.zeros_like(code), code).flatten(-2), torch.where(bad, torch.full_like(e, 128), e) + 127


def pack(code):
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8)


def unpack(packed):
    p = packed.cpu()
    return torch.stack([p & 15, p >> 4], -1).flatten(-2)


def values(packed, exponents):
    """What a 4-bit cache's rows stand for."""
    code = unpack(packed).long()
    size = LEVELS[code & 7] * torch.where(code >= 8, -1.0, 1.0).double()
    e = exponents.cpu().double()
    power = torch.where(e == 255, torch.full_like(e, math.nan), torch.pow(2.0, e - 127))
    return size * power.repeat_interleave(32, -1)


def margin(x, error, dtype):
    """Whether each x is nearer than `error` to where its code or its block's exponent changes."""
    low, high = POWERS[dtype]
    top, where = x.abs().unflatten(-1, (-1, 32)).max(-1)
    slack = error.unflatten(-1, (-1, 32)).amax(-1)
    near = torch.zeros(top.shape, dtype=torch.bool)
    for i in range(low, high):
        near |= (top - 6.0 * 2.0 ** i).abs() <= slack
    _, e = blocks(x, dtype)
    s = torch.pow(2.0, e.double() - 127).repeat_interleave(32, -1)
    close = near.repeat_interleave(32, -1)
    for i in range(7):
        close |= (x.abs() - s * (LEVELS[i] + LEVELS[i + 1]) / 2).abs() <= error
    return close


def cut_cache(x, dtype):
    """x [pages, heads, page, d] on the GPU as a 4-bit cache there: codes and exponents."""
    code, e = blocks(x.cpu().double(), dtype)
    return pack(code).to(x.device), e.to(torch.uint8).to(x.device)


def attend(q, k_cache, v_cache, table, lengths, window=0, scale=None, k_scale=None, v_scale=None):
    """out, lse, sum of p |v| as serving_ref has them, and the masses added, [batch, heads, longest]."""
    if k_cache.dtype == torch.uint8:
        k_cache, v_cache, k_scale, v_scale = values(k_cache, k_scale), values(v_cache, v_scale), None, None
    out, lse, size = ref.attend(q, k_cache, v_cache, table, lengths, window, scale, k_scale, v_scale)
    batch, hq, d = q.shape
    hk, page = k_cache.shape[1], k_cache.shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    mass = torch.zeros(batch, hk, max(1, int(lengths.max())), dtype=torch.float64)
    for b in range(batch):
        n = int(lengths[b])
        lo = max(0, n - window) if window else 0
        if n <= lo:
            continue
        at = torch.arange(lo, n)
        pages, off = table[b].cpu().long()[at // page].to(k_cache.device), (at % page).to(k_cache.device)
        for h in range(hq):
            kh = h // (hq // hk)
            k = ref.d64(ref._rows(k_cache, pages, kh, off))
            if k_scale is not None:
                k = k * float(k_scale[kh])
            s = (k * ref.d64(q)[b, h]).sum(1) * scale
            p = torch.softmax(s, 0)
            if not bool((s == -math.inf).all()):
                mass[b, kh, lo:n] += p
    return out, lse, size, mass


def evict(mass, n, keep, recent, sink):
    """Which token is at each place afterwards: masses of one sequence and head (a list), its length."""
    if n <= keep:
        return list(range(n))
    safe = set(range(sink)) | set(range(n - recent, n))

    def rank(j):
        m = mass[j]
        return (1, 0.0, j) if math.isnan(m) else (0, -m, j)

    others = sorted((j for j in range(n) if j not in safe), key=rank)
    stay = safe | set(others[:keep - len(safe)])
    front = keep - recent
    movers = iter(sorted(j for j in stay if front <= j < n - recent))
    return [j if j in stay else next(movers) for j in range(front)] + list(range(n - recent, n))
