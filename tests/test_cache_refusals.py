"""Arguments that the operators that keep a session's cache small refuse, at the C-ABI (before
anything is enqueued, so no GPU is needed) and in the binding."""
import ctypes
import math
import os

import pytest

torch = pytest.importorskip("torch")

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16, F16, E4M3, E2M1 = 0, 1, 2, 3, 4


def _at(i):
    """Addresses 2^36 apart, aligned, never dereferenced by the host checks."""
    return ctypes.c_void_p((i + 1) << 36)


FAKE, ODD = _at(0), ctypes.c_void_p((1 << 36) + 8)


@pytest.fixture(scope="module")
def lib():
    import paper_2608_13226_amd as cp
    if not os.path.exists(cp.library_path()):
        from paper_2608_13226_amd import build
        build.build()
    return cp.library()


def _append(lib, **kw):
    a = dict(q=_at(1), q_stride=1024, k=_at(2), k_stride=256, v=_at(3), v_stride=256, dtype=BF16, tokens=3, hq=8, hk=2, d=128,
             positions=FAKE, slots=FAKE, inv_freq=FAKE, rot=128, interleaved=0, magnitude=1.0, q_out=_at(4), k_cache=_at(5),
             v_cache=_at(6), pages=10, page_size=16, k_scale=FAKE, v_scale=FAKE, stream=None)
    a.update(kw)
    return lib.coverprune_kv_append4(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), INVALID), (dict(tokens=1 << 31), INVALID), (dict(hq=0), INVALID), (dict(hk=0), INVALID), (dict(d=0), UNSUPPORTED),
    (dict(d=48), UNSUPPORTED), (dict(d=4128), UNSUPPORTED), (dict(rot=3), INVALID), (dict(rot=-2), INVALID), (dict(rot=130), INVALID),
    (dict(page_size=0), INVALID), (dict(page_size=(1 << 20) + 1), INVALID), (dict(pages=0), INVALID), (dict(dtype=F32), UNSUPPORTED),
    (dict(dtype=E2M1), UNSUPPORTED), (dict(magnitude=math.nan), INVALID), (dict(magnitude=-1e39), INVALID), (dict(q_stride=1000), INVALID), (dict(k_stride=255), INVALID),
    (dict(v_stride=0), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(positions=None), INVALID),
    (dict(slots=None), INVALID), (dict(inv_freq=None), INVALID), (dict(q_out=None), INVALID), (dict(k_cache=None), INVALID),
    (dict(v_cache=None), INVALID), (dict(k_scale=None), INVALID), (dict(v_scale=None), INVALID), (dict(k_cache=ODD), INVALID),
    (dict(q_out=ODD), INVALID), (dict(q_out=_at(1)), INVALID), (dict(q_out=ctypes.c_void_p((2 << 36) + 3 * 2048 - 16)), INVALID),
    (dict(q_out=_at(2)), INVALID), (dict(q_out=ctypes.c_void_p((4 << 36) - 3 * 2048 + 16)), INVALID)])
def test_append4_rejects(lib, kw, code):
    assert _append(lib, **kw) == code and lib.coverprune_last_error() != b""


def _gather(lib, **kw):
    a = dict(k_cache=FAKE, v_cache=FAKE, cache_dtype=BF16, pages=10, page_size=16, hk=2, d=128, k_scale=None, v_scale=None, slots=FAKE,
             tokens=5, k_out=FAKE, v_out=FAKE, dtype=BF16, stream=None)
    a.update(kw)
    return lib.coverprune_kv_gather(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), INVALID), (dict(tokens=1 << 31), INVALID), (dict(hk=0), INVALID), (dict(d=0), INVALID), (dict(d=4097), INVALID),
    (dict(page_size=0), INVALID), (dict(pages=0), INVALID), (dict(dtype=F32), UNSUPPORTED), (dict(dtype=E4M3), UNSUPPORTED),
    (dict(cache_dtype=F16), UNSUPPORTED), (dict(cache_dtype=F32), UNSUPPORTED), (dict(cache_dtype=9), UNSUPPORTED),
    (dict(cache_dtype=E2M1, d=100, k_scale=FAKE, v_scale=FAKE), UNSUPPORTED), (dict(k_scale=FAKE), INVALID), (dict(v_scale=FAKE), INVALID),
    (dict(cache_dtype=E2M1), INVALID), (dict(cache_dtype=E2M1, k_scale=FAKE), INVALID), (dict(k_cache=None), INVALID),
    (dict(v_cache=None), INVALID), (dict(slots=None), INVALID), (dict(k_out=None), INVALID), (dict(v_out=None), INVALID),
    (dict(k_cache=ODD), INVALID), (dict(v_out=ODD), INVALID)])
def test_gather_rejects(lib, kw, code):
    assert _gather(lib, **kw) == code and lib.coverprune_last_error() != b""


def _attend4(lib, **kw):
    a = dict(q=FAKE, dtype=BF16, batch=2, hq=8, hk=2, d=128, k_cache=FAKE, v_cache=FAKE, pages=100, page_size=16, k_scale=FAKE,
             v_scale=FAKE, table=FAKE, width=10, lengths=FAKE, max_length=160, window=0, scale=0.1, out=FAKE, lse=None, ws=None,
             ws_bytes=0, stream=None)
    a.update(kw)
    return lib.coverprune_paged_attention4(*a.values())


def _mass(lib, **kw):
    a = dict(q=FAKE, dtype=BF16, batch=2, hq=8, hk=2, d=128, k_cache=FAKE, v_cache=FAKE, cache_dtype=BF16, pages=100, page_size=16,
             k_scale=None, v_scale=None, table=FAKE, width=10, lengths=FAKE, max_length=160, window=0, scale=0.1, mass=FAKE, mass_span=160,
             out=FAKE, lse=None, ws=None, ws_bytes=0, stream=None)
    a.update(kw)
    return lib.coverprune_paged_attention_mass(*a.values())


COMMON = [
    (dict(batch=-1), INVALID), (dict(batch=65536), INVALID), (dict(hq=7), INVALID), (dict(hk=0), INVALID), (dict(hq=0), INVALID),
    (dict(d=80), UNSUPPORTED), (dict(d=0), UNSUPPORTED), (dict(max_length=0), INVALID), (dict(max_length=161), INVALID),
    (dict(max_length=1 << 31, width=1 << 27), INVALID), (dict(window=-1), INVALID), (dict(dtype=F32), UNSUPPORTED),
    (dict(dtype=E2M1), UNSUPPORTED), (dict(page_size=0), INVALID), (dict(pages=0), UNSUPPORTED), (dict(pages=1 << 28), UNSUPPORTED),
    (dict(width=0), INVALID), (dict(width=1 << 28), INVALID), (dict(scale=math.inf), INVALID), (dict(q=None), INVALID),
    (dict(k_cache=None), INVALID), (dict(v_cache=None), INVALID), (dict(table=None), INVALID), (dict(lengths=None), INVALID),
    (dict(out=None), INVALID), (dict(q=ODD), INVALID), (dict(out=ODD), INVALID), (dict(v_cache=ODD), INVALID)]


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(k_scale=None), INVALID), (dict(v_scale=None), INVALID), (dict(width=10000, max_length=160000), WORKSPACE),
    (dict(width=10000, max_length=160000, ws=FAKE, ws_bytes=64), WORKSPACE)])
def test_attention4_rejects(lib, kw, code):
    assert _attend4(lib, **kw) == code and lib.coverprune_last_error() != b""


LONG = dict(width=10000, max_length=160000, mass_span=160000)


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(cache_dtype=F16), UNSUPPORTED), (dict(cache_dtype=F32), UNSUPPORTED), (dict(k_scale=FAKE), INVALID),
    (dict(cache_dtype=E2M1), INVALID), (dict(cache_dtype=E2M1, k_scale=FAKE), INVALID), (dict(mass=None), INVALID),
    (dict(mass_span=159), INVALID), (dict(mass_span=1 << 31), INVALID), (LONG, WORKSPACE),
    (dict(LONG, ws=FAKE, ws_bytes=2 * 8 * 160000 * 4), WORKSPACE),
    # More blocks for the join than a launch has.
    (dict(batch=65535, hq=65535, hk=1), UNSUPPORTED)])
def test_mass_rejects(lib, kw, code):
    assert _mass(lib, **kw) == code and lib.coverprune_last_error() != b""


def _evict(lib, **kw):
    a = dict(k_cache=FAKE, v_cache=FAKE, cache_dtype=BF16, pages=100, page_size=16, hk=2, d=128, k_scale=None, v_scale=None, table=FAKE,
             batch=2, width=10, lengths=_at(1), max_length=160, mass=_at(2), mass_span=160, keep=100, recent=10, sink=4, kept=FAKE,
             mass_out=_at(2), lengths_out=_at(3), ws=None, ws_bytes=0, stream=None)
    a.update(kw)
    return lib.coverprune_kv_evict(*a.values())


BIG = dict(width=10000, max_length=160000, mass_span=160000, keep=80000)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), INVALID), (dict(batch=65536), INVALID), (dict(hk=0), INVALID), (dict(hk=65536), INVALID), (dict(keep=0), INVALID),
    (dict(keep=-1), INVALID), (dict(keep=1 << 31), INVALID), (dict(recent=-1), INVALID), (dict(recent=101), INVALID),
    (dict(sink=-1), INVALID), (dict(sink=91), INVALID), (dict(recent=2 ** 62, sink=2 ** 62), INVALID), (dict(max_length=0), INVALID),
    (dict(max_length=161), INVALID), (dict(max_length=(1 << 31) - 2048, width=1 << 27), INVALID), (dict(mass_span=159), INVALID),
    (dict(max_length=(1 << 30) + 1, width=1 << 27, mass_span=(1 << 30) + 1), INVALID), (dict(batch=65535, hk=257), UNSUPPORTED),
    (dict(mass_span=1 << 31), INVALID), (dict(page_size=0), INVALID), (dict(pages=0), UNSUPPORTED), (dict(pages=1 << 28), UNSUPPORTED),
    (dict(width=0), INVALID), (dict(cache_dtype=F32), UNSUPPORTED), (dict(cache_dtype=9), UNSUPPORTED), (dict(d=0), UNSUPPORTED),
    (dict(d=4), UNSUPPORTED), (dict(d=100), UNSUPPORTED), (dict(d=4104), UNSUPPORTED), (dict(cache_dtype=E2M1, d=40), UNSUPPORTED),
    (dict(k_scale=FAKE), INVALID), (dict(cache_dtype=E4M3, v_scale=FAKE), INVALID), (dict(cache_dtype=E2M1), INVALID),
    (dict(k_cache=None), INVALID), (dict(v_cache=None), INVALID), (dict(table=None), INVALID), (dict(lengths=None), INVALID),
    (dict(mass=None), INVALID), (dict(kept=None), INVALID), (dict(mass_out=None), INVALID), (dict(lengths_out=None), INVALID),
    (dict(lengths_out=_at(1)), INVALID), (dict(lengths_out=ctypes.c_void_p((2 << 36) + 4)), INVALID),
    (dict(mass_out=ctypes.c_void_p((3 << 36) + 1276)), INVALID), (dict(k_cache=ODD), INVALID), (BIG, WORKSPACE),
    (dict(BIG, ws=FAKE, ws_bytes=1000), WORKSPACE), (dict(BIG, ws=ODD, ws_bytes=1 << 30), WORKSPACE)])
def test_evict_rejects(lib, kw, code):
    assert _evict(lib, **kw) == code and lib.coverprune_last_error() != b""


def test_nothing_to_do_is_fine(lib):
    assert _append(lib, tokens=0, k=None) == OK and _gather(lib, tokens=0, slots=None) == OK
    assert _attend4(lib, batch=0, q=None) == OK and _mass(lib, batch=0, q=None) == OK and _evict(lib, batch=0, mass=None) == OK


def test_workspaces(lib):
    size, mass, evict = (lib.coverprune_paged_attention_workspace, lib.coverprune_paged_attention_mass_workspace,
                         lib.coverprune_kv_evict_workspace)
    for bad in ((-1, 8, 2, 128, 100, 0), (1, 7, 2, 128, 100, 0), (1, 8, 2, 80, 100, 0), (1, 8, 2, 128, 0, 0), (1, 8, 2, 128, 100, -1)):
        assert mass(*bad) == 0
    assert mass(1, 28, 4, 128, 1, 0) == 0
    # The scores beside what the other call takes.
    for case in ((1, 28, 4, 128, 131072, 0), (16, 28, 4, 128, 65536, 0), (3, 40, 2, 64, 500, 0), (2, 20, 1, 256, 600, 100)):
        assert mass(*case) >= size(*case) + 4 * case[0] * case[1] * min(case[4], case[5] or case[4])
    for bad in ((-1, 2, 10, 1, 100), (1, 0, 10, 1, 100), (1, 2, 0, 0, 100), (1, 2, 10, 11, 100), (1, 2, 10, -1, 100), (1, 2, 10, 1, 0),
                (1, 2, 10, 1, (1 << 30) + 1), (65535, 65535, 1 << 29, 0, 1 << 30)):
        assert evict(*bad) == 0
    assert evict(4, 2, 100, 10, 90) == 0
    assert evict(1, 1, 50000, 100, 100000) >= 4 * (2 * 49900 + 50000)


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


U8, F, I32, I64, EIGHT = torch.uint8, torch.float32, torch.int32, torch.int64, torch.float8_e4m3fn


def _good():
    """Each operator's arguments in order, on the CPU."""
    import paper_2608_13226_amd as cp
    q, k = _t(3, 8, 128), _t(3, 2, 128)
    c4, s4 = _t(4, 2, 16, 64, dtype=U8), _t(4, 2, 16, 4, dtype=U8)
    table, n = _t(3, 2, dtype=I32), _t(3, dtype=I32)
    return {
        "append": (cp.kv_append4, dict(q=q, k=k, v=k.clone(), positions=_t(3, dtype=I32), slots=_t(3, dtype=I64), inv_freq=_t(64, dtype=F),
                                       k_cache=c4, v_cache=c4.clone(), k_scale=s4, v_scale=s4.clone(), q_out=q.clone())),
        "gather": (cp.kv_gather, dict(k_cache=c4, v_cache=c4.clone(), slots=_t(5, dtype=I64), k_scale=s4, v_scale=s4.clone(),
                                      k_out=_t(5, 2, 128), v_out=_t(5, 2, 128))),
        "gather16": (cp.kv_gather, dict(k_cache=_t(4, 2, 16, 128), v_cache=_t(4, 2, 16, 128), slots=_t(5, dtype=I64))),
        "attend": (cp.paged_attention4, dict(q=q, k_cache=c4, v_cache=c4.clone(), k_scale=s4, v_scale=s4.clone(), table=table, lengths=n,
                                             out=q.clone(), lse=_t(3, 8, dtype=F), max_length=32)),
        "mass": (cp.paged_attention_mass, dict(q=q, k_cache=_t(4, 2, 16, 128), v_cache=_t(4, 2, 16, 128), table=table, lengths=n,
                                               mass=_t(3, 2, 40, dtype=F), out=q.clone(), lse=_t(3, 8, dtype=F), max_length=32)),
        "mass8": (cp.paged_attention_mass, dict(q=q, k_cache=_t(4, 2, 16, 128).to(EIGHT), v_cache=_t(4, 2, 16, 128).to(EIGHT), table=table,
                                                lengths=n, mass=_t(3, 2, 40, dtype=F), k_scale=_t(2, dtype=F), v_scale=_t(2, dtype=F))),
        "evict": (cp.kv_evict, dict(k_cache=_t(4, 2, 16, 128), v_cache=_t(4, 2, 16, 128), table=table, lengths=n,
                                    mass=_t(3, 2, 40, dtype=F), keep=10, recent=2, sink=1, kept=_t(3, 2, 10, dtype=I32),
                                    mass_out=_t(3, 2, 40, dtype=F), lengths_out=n.clone())),
        "evict4": (cp.kv_evict, dict(k_cache=c4, v_cache=c4.clone(), k_scale=s4, v_scale=s4.clone(), table=table, lengths=n,
                                     mass=_t(3, 2, 40, dtype=F), keep=10))}


NAMES = ["append", "gather", "gather16", "attend", "mass", "mass8", "evict", "evict4"]


@pytest.mark.parametrize("which", NAMES)
def test_only_the_gpu_is_missing(which):
    f, a = _good()[which]
    with pytest.raises(ValueError, match="GPU"):
        f(**a)


@pytest.mark.parametrize("which,bad,err", [
    ("append", dict(q=_t(3, 8, 128, dtype=F)), TypeError), ("append", dict(q=_t(3, 128, 8).transpose(1, 2)), ValueError),
    ("append", dict(k=_t(3, 2, 64)), ValueError), ("append", dict(v=_t(3, 4, 128)), ValueError),
    ("append", dict(positions=_t(3, dtype=I64)), TypeError), ("append", dict(slots=_t(3, dtype=I32)), TypeError),
    ("append", dict(inv_freq=_t(64)), TypeError), ("append", dict(k_cache=_t(4, 2, 16, 128)), TypeError),
    ("append", dict(v_cache=_t(4, 2, 16, 32, dtype=U8)), ValueError), ("append", dict(k_scale=_t(4, 2, 16, 2, dtype=U8)), ValueError),
    ("append", dict(v_scale=_t(2, dtype=F)), TypeError), ("append", dict(k_scale=None), TypeError),
    ("append", dict(k=_t(3, 3, 128), v=_t(3, 3, 128)), ValueError), ("append", dict(q_out=_t(3, 8, 64)), ValueError),
    ("gather", dict(slots=_t(5, dtype=I32)), TypeError), ("gather", dict(slots=_t(5, 1, dtype=I64)), ValueError),
    ("gather", dict(dtype=F), TypeError), ("gather", dict(k_scale=None), ValueError), ("gather", dict(v_out=_t(5, 2, 64)), ValueError),
    ("gather", dict(dtype=torch.float16), TypeError), ("gather16", dict(dtype=torch.float16), TypeError),
    ("gather16", dict(k_scale=_t(2, dtype=F)), ValueError), ("gather16", dict(v_cache=_t(4, 2, 16, 64)), ValueError),
    ("gather16", dict(k_cache=_t(4, 2, 16, 128, dtype=F)), TypeError),
    ("attend", dict(q=_t(3, 8, 64)), ValueError), ("attend", dict(q=_t(3, 8, 128, dtype=F)), TypeError),
    ("attend", dict(k_cache=_t(4, 2, 16, 128)), TypeError), ("attend", dict(k_scale=_t(4, 2, 16, 64, dtype=U8)), ValueError),
    ("attend", dict(table=_t(3, 2, dtype=I64)), TypeError), ("attend", dict(lengths=_t(2, dtype=I32)), ValueError),
    ("attend", dict(max_length="long"), TypeError), ("attend", dict(scale="big"), TypeError), ("attend", dict(lse=_t(3, 8)), TypeError),
    ("mass", dict(mass=_t(3, 2, 40)), TypeError), ("mass", dict(mass=_t(3, 4, 40, dtype=F)), ValueError),
    ("mass", dict(mass=_t(3, 2, 80, dtype=F)[:, :, ::2]), ValueError), ("mass", dict(k_scale=_t(2, dtype=F)), ValueError),
    ("mass", dict(k_cache=_t(4, 2, 16, 128).half(), v_cache=_t(4, 2, 16, 128).half()), TypeError), ("mass", dict(mass=None), TypeError),
    ("mass8", dict(k_scale=_t(4, 2, 16, 4, dtype=U8)), TypeError), ("mass8", dict(k_cache=_t(4, 2, 16, 128)), TypeError),
    ("evict", dict(mass=_t(3, 2, 40)), TypeError), ("evict", dict(keep=0), ValueError), ("evict", dict(keep=2.5), TypeError),
    ("evict", dict(kept=_t(3, 2, 9, dtype=I32)), ValueError), ("evict", dict(k_scale=_t(2, dtype=F)), ValueError),
    ("evict", dict(lengths=_t(3, dtype=I64)), TypeError), ("evict", dict(table=_t(6, dtype=I32)), ValueError),
    ("evict", dict(lengths_out=_t(4, dtype=I32)), ValueError), ("evict", dict(k_cache=_t(4, 2, 128, 16).transpose(2, 3)), ValueError),
    ("evict4", dict(k_scale=None), ValueError), ("evict4", dict(v_scale=_t(4, 2, 16, 64, dtype=U8)), ValueError),
    ("evict4", dict(mass=_t(3, 40, dtype=F)), ValueError)])
def test_binding_refuses(which, bad, err):
    f, a = _good()[which]
    with pytest.raises(err) as e:
        f(**{**a, **bad})
    assert "GPU" not in str(e.value)


def test_eight_bit_caches_evict_without_scales():
    f, a = _good()["evict"]
    a.update(k_cache=_t(4, 2, 16, 128).to(EIGHT), v_cache=_t(4, 2, 16, 128).to(EIGHT))
    with pytest.raises(ValueError, match="GPU"):
        f(**a)
    with pytest.raises(ValueError, match="4-bit"):
        f(**a, k_scale=_t(2, dtype=F))


@pytest.mark.parametrize("which", NAMES)
def test_no_gradient_is_cut_off(which):
    """A tensor that requires a gradient is refused, unless none are asked for."""
    f, a = _good()[which]
    for name, t in a.items():
        if not isinstance(t, torch.Tensor) or not t.is_floating_point():
            continue
        wants = t.detach().clone().requires_grad_()
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            f(**{**a, name: wants})
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            f(**{**a, name: wants})
