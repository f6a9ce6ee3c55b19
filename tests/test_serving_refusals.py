"""Arguments that the serving operators refuse, at the C-ABI (before anything
is enqueued, so no GPU is needed) and in the binding."""
import ctypes
import math
import os

import pytest

torch = pytest.importorskip("torch")

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16, F16, E4M3 = 0, 1, 2, 3
FAKE = ctypes.c_void_p(0x1000)          # aligned, never dereferenced by the host checks
ODD = ctypes.c_void_p(0x1008)


@pytest.fixture(scope="module")
def lib():
    import paper_2608_13226_amd as cp
    if not os.path.exists(cp.library_path()):
        from paper_2608_13226_amd import build
        build.build()
    return cp.library()


def _norm(lib, **kw):
    a = dict(x=FAKE, dtype=BF16, rows=4, d=64, residual=None, weight=FAKE, eps=1e-6, out=FAKE, out_dtype=BF16, out_scale=None,
             residual_out=None, stream=None)
    a.update(kw)
    return lib.coverprune_rms_norm(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), INVALID), (dict(rows=1 << 31), INVALID), (dict(d=0), INVALID), (dict(d=65537), INVALID),
    (dict(dtype=E4M3), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED), (dict(out_dtype=F16), UNSUPPORTED),
    (dict(eps=-1.0), INVALID), (dict(eps=math.nan), INVALID), (dict(x=None), INVALID), (dict(weight=None), INVALID),
    (dict(out=None), INVALID), (dict(residual=FAKE), INVALID), (dict(out_dtype=E4M3), INVALID), (dict(x=ODD), INVALID),
    (dict(weight=ODD), INVALID), (dict(out=ODD), INVALID), (dict(residual=ODD, residual_out=FAKE), INVALID),
    (dict(residual=FAKE, residual_out=ODD), INVALID)])
def test_norm_rejects(lib, kw, code):
    assert _norm(lib, **kw) == code and lib.coverprune_last_error() != b""


def _w4(lib, **kw):
    a = dict(x=FAKE, x_dtype=BF16, x_scale=None, weight=FAKE, scale=FAKE, zero=None, m=2, n=32, k=256, group=128, dtype=BF16,
             y=FAKE, y_dtype=BF16, stream=None)
    a.update(kw)
    return lib.coverprune_w4_matvec(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(m=-1), INVALID), (dict(m=(1 << 20) + 1), INVALID), (dict(n=0), INVALID), (dict(n=1 << 31), INVALID), (dict(k=0), INVALID),
    (dict(k=(1 << 20) + 32), INVALID), (dict(group=0), UNSUPPORTED), (dict(group=16), UNSUPPORTED), (dict(group=48), UNSUPPORTED),
    (dict(group=96), UNSUPPORTED), (dict(dtype=F32), UNSUPPORTED), (dict(x_dtype=F16), UNSUPPORTED), (dict(y_dtype=F16), UNSUPPORTED),
    (dict(y_dtype=E4M3), UNSUPPORTED), (dict(x_scale=FAKE), INVALID), (dict(x_dtype=E4M3), INVALID), (dict(x=None), INVALID),
    (dict(weight=None), INVALID), (dict(scale=None), INVALID), (dict(y=None), INVALID), (dict(x=ODD), INVALID),
    (dict(weight=ODD), INVALID)])
def test_w4_rejects(lib, kw, code):
    assert _w4(lib, **kw) == code and lib.coverprune_last_error() != b""


def _append(lib, **kw):
    a = dict(q=FAKE, q_stride=1024, k=FAKE, k_stride=256, v=FAKE, v_stride=256, dtype=BF16, tokens=3, hq=8, hk=2, d=128,
             positions=FAKE, slots=FAKE, inv_freq=FAKE, rot=128, interleaved=0, magnitude=1.0, q_out=FAKE, k_cache=FAKE, v_cache=FAKE,
             cache_dtype=BF16, pages=10, page_size=16, k_scale=None, v_scale=None, stream=None)
    a.update(kw)
    return lib.coverprune_kv_append(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), INVALID), (dict(hq=0), INVALID), (dict(hk=0), INVALID), (dict(d=0), INVALID), (dict(d=5000), INVALID),
    (dict(rot=3), INVALID), (dict(rot=-2), INVALID), (dict(rot=130), INVALID), (dict(page_size=0), INVALID), (dict(pages=0), INVALID),
    (dict(dtype=F32), UNSUPPORTED), (dict(cache_dtype=F16), UNSUPPORTED), (dict(cache_dtype=F32), UNSUPPORTED),
    (dict(k_scale=FAKE), INVALID), (dict(v_scale=FAKE), INVALID), (dict(magnitude=math.inf), INVALID), (dict(q_stride=1000), INVALID),
    (dict(k_stride=255), INVALID), (dict(v_stride=0), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(positions=None), INVALID), (dict(slots=None), INVALID), (dict(inv_freq=None), INVALID), (dict(q_out=None), INVALID),
    (dict(k_cache=None), INVALID), (dict(v_cache=None), INVALID), (dict(k_cache=ODD), INVALID), (dict(q_out=ODD), INVALID)])
def test_append_rejects(lib, kw, code):
    assert _append(lib, **kw) == code and lib.coverprune_last_error() != b""


def _attend(lib, **kw):
    a = dict(q=FAKE, dtype=BF16, batch=2, hq=8, hk=2, d=128, k_cache=FAKE, v_cache=FAKE, cache_dtype=BF16, pages=100, page_size=16,
             k_scale=None, v_scale=None, table=FAKE, width=10, lengths=FAKE, max_length=160, window=0, scale=0.1, out=FAKE, lse=None,
             ws=None, ws_bytes=0, stream=None)
    a.update(kw)
    return lib.coverprune_paged_attention(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), INVALID), (dict(batch=65536), INVALID), (dict(hq=7), INVALID), (dict(hk=0), INVALID), (dict(hq=0), INVALID),
    (dict(d=80), UNSUPPORTED), (dict(d=0), UNSUPPORTED), (dict(max_length=0), INVALID), (dict(max_length=161), INVALID),
    (dict(max_length=1 << 31, width=1 << 27), INVALID), (dict(window=-1), INVALID), (dict(dtype=F32), UNSUPPORTED),
    (dict(cache_dtype=F16), UNSUPPORTED), (dict(k_scale=FAKE), INVALID), (dict(page_size=0), INVALID), (dict(pages=0), UNSUPPORTED),
    (dict(pages=1 << 28), UNSUPPORTED), (dict(width=0), INVALID), (dict(width=1 << 28), INVALID), (dict(scale=math.nan), INVALID),
    (dict(q=None), INVALID), (dict(k_cache=None), INVALID), (dict(v_cache=None), INVALID), (dict(table=None), INVALID),
    (dict(lengths=None), INVALID), (dict(out=None), INVALID), (dict(q=ODD), INVALID), (dict(out=ODD), INVALID),
    (dict(width=10000, max_length=160000), WORKSPACE), (dict(width=10000, max_length=160000, ws=FAKE, ws_bytes=64), WORKSPACE),
    (dict(width=10000, max_length=160000, ws=ODD, ws_bytes=1 << 30), WORKSPACE)])
def test_attention_rejects(lib, kw, code):
    assert _attend(lib, **kw) == code and lib.coverprune_last_error() != b""


def test_nothing_to_do_is_fine(lib):
    """Counts of 0 enqueue nothing and succeed, whatever the pointers."""
    assert _norm(lib, rows=0, x=None) == OK and _w4(lib, m=0, x=None) == OK
    assert _append(lib, tokens=0, k=None) == OK and _attend(lib, batch=0, q=None) == OK


def test_attention_workspace(lib):
    size = lib.coverprune_paged_attention_workspace
    for bad in ((-1, 8, 2, 128, 100, 0), (1, 7, 2, 128, 100, 0), (1, 8, 2, 80, 100, 0), (1, 8, 2, 128, 0, 0), (1, 8, 2, 128, 100, -1)):
        assert size(*bad) == 0
    assert size(1, 28, 4, 128, 1, 0) == 0
    assert size(1, 28, 4, 128, 131072, 0) >= 28 * 128 * 4 * 2
    # A window bounds what there is to cut.
    assert size(1, 28, 4, 128, 131072, 32) == 0


@pytest.mark.parametrize("window", [131072, 2 ** 31, 2 ** 62, 2 ** 63 - 33, 2 ** 63 - 32, 2 ** 63 - 1])
def test_a_window_past_the_longest_length_is_none(lib, window):
    """Any window of 64 bits: the workspace is that of the runs that are then written."""
    size = lib.coverprune_paged_attention_workspace
    assert size(1, 28, 4, 128, 131072, window) == size(1, 28, 4, 128, 131072, 0)
    assert _attend(lib, width=10000, max_length=160000, window=window) == WORKSPACE


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def test_binding_refuses():
    import paper_2608_13226_amd as cp
    x, w = _t(4, 64), _t(64)
    with pytest.raises(TypeError):
        cp.rms_norm(_t(4, 64, dtype=torch.float64), w)
    with pytest.raises(TypeError):
        cp.rms_norm(x, _t(64, dtype=torch.float16))
    with pytest.raises(ValueError):
        cp.rms_norm(x, _t(65))
    with pytest.raises(ValueError):
        cp.rms_norm(_t(64), w)
    with pytest.raises(ValueError, match="contiguous"):
        cp.rms_norm(_t(64, 4).t(), w)
    with pytest.raises(ValueError):
        cp.rms_norm(x, w, residual=_t(5, 64))
    with pytest.raises(TypeError):
        cp.rms_norm(x, w, quantize=True, out=_t(4, 64))

    x, cw, s = _t(2, 256), _t(32, 128, dtype=torch.uint8), _t(32, 2)
    with pytest.raises(ValueError):
        cp.w4_matvec(x, _t(32, 64, dtype=torch.uint8), s)
    with pytest.raises(TypeError):
        cp.w4_matvec(x, cw.to(torch.int32), s)
    with pytest.raises(TypeError):
        cp.w4_matvec(x.half(), cw, s)
    with pytest.raises(ValueError):
        cp.w4_matvec(x, cw, _t(32, 3))
    with pytest.raises(ValueError, match="x_scale"):
        cp.w4_matvec(x.to(torch.float8_e4m3fn), cw, s)
    with pytest.raises(TypeError):
        cp.w4_matvec(x, cw, s, out_dtype=torch.float16)

    q, k = _t(3, 8, 128), _t(3, 2, 128)
    pos, slots, inv = _t(3, dtype=torch.int32), _t(3, dtype=torch.int64), _t(64, dtype=torch.float32)
    cache = _t(4, 2, 16, 128)
    good = [q, k, k, pos, slots, inv, cache, cache]
    for i, bad, err in ((0, q.float(), TypeError), (0, _t(3, 128, 8).transpose(1, 2), ValueError), (1, _t(3, 2, 64), ValueError),
                        (2, _t(3, 4, 128), ValueError), (2, _t(2, 2, 128), ValueError), (3, pos.long(), TypeError), (4, slots.int(), TypeError),
                        (5, inv.double(), TypeError), (6, cache.half(), TypeError), (7, _t(4, 2, 16, 64), ValueError),
                        (0, _t(1, 8, 128).expand(3, 8, 128), ValueError)):
        args = list(good)
        args[i] = bad
        with pytest.raises(err):
            cp.kv_append(*args)
    with pytest.raises(ValueError):
        cp.kv_append(*good, k_scale=_t(2, dtype=torch.float32))

    table, n = _t(3, 2, dtype=torch.int32), _t(3, dtype=torch.int32)
    good = [q, cache, cache, table, n]
    for i, bad, err in ((0, q.float(), TypeError), (0, q[:2], ValueError), (1, cache.half(), TypeError), (2, _t(5, 2, 16, 128), ValueError),
                        (3, table.long(), TypeError), (4, n.long(), TypeError), (4, _t(2, dtype=torch.int32), ValueError)):
        args = list(good)
        args[i] = bad
        with pytest.raises(err):
            cp.paged_attention(*args)
    # Everything else in order, but not on the GPU.
    with pytest.raises(ValueError, match="GPU"):
        cp.paged_attention(*good, max_length=32)
    with pytest.raises(ValueError, match="GPU"):
        cp.rms_norm(_t(4, 64), w)


def _calls():
    """Each operator with its tensors by name, on the CPU and otherwise in order."""
    import paper_2608_13226_amd as cp
    f32, e4m3 = torch.float32, torch.float8_e4m3fn
    q, k, cache = _t(3, 8, 128), _t(3, 2, 128), _t(4, 2, 16, 128).to(e4m3)
    scales = dict(k_scale=_t(2, dtype=f32), v_scale=_t(2, dtype=f32))
    return [
        (cp.rms_norm, dict(x=_t(4, 64), weight=_t(64), residual=_t(4, 64), out=_t(4, 64), residual_out=_t(4, 64)), {}),
        (cp.w4_matvec, dict(x=_t(2, 256), weight=_t(32, 128, dtype=torch.uint8), scale=_t(32, 2), out=_t(2, 32)), {}),
        (cp.w4_matvec, dict(x=_t(2, 256).to(e4m3), weight=_t(32, 128, dtype=torch.uint8), scale=_t(32, 2), x_scale=_t(2, dtype=f32)), {}),
        (cp.kv_append, dict(q=q, k=k, v=k.clone(), positions=_t(3, dtype=torch.int32), slots=_t(3, dtype=torch.int64),
                            inv_freq=_t(64, dtype=f32), k_cache=cache, v_cache=cache.clone(), q_out=q.clone(), **scales), {}),
        (cp.paged_attention, dict(q=q, k_cache=cache, v_cache=cache.clone(), table=_t(3, 2, dtype=torch.int32),
                                  lengths=_t(3, dtype=torch.int32), out=q.clone(), lse=_t(3, 8, dtype=f32), **scales),
         dict(max_length=32, return_lse=True))]


@pytest.mark.parametrize("i", range(5))
def test_no_gradient_is_cut_off(i):
    """A tensor that requires a gradient is refused, unless none are asked for."""
    f, tensors, rest = _calls()[i]
    with pytest.raises(ValueError, match="GPU"):
        f(**tensors, **rest)
    for name, t in tensors.items():
        if not t.is_floating_point():
            continue
        wants = t.detach().clone().requires_grad_()
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            f(**{**tensors, name: wants}, **rest)
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            f(**{**tensors, name: wants}, **rest)


@pytest.mark.parametrize("version,match", [(2, "older than this binding.*rebuild"), (1, "ABI 1.*rebuild")])
def test_a_library_built_before_these_operators(monkeypatch, tmp_path, version, match):
    """One that lacks entry points is named as such, whatever is called first; another ABI is said to be one."""
    import subprocess
    import paper_2608_13226_amd as cp
    src, lib = tmp_path / "old.c", tmp_path / f"libold{version}.so"
    src.write_text(f"int coverprune_abi_version(void) {{ return {version}; }}\n")
    subprocess.run(["gcc", "-shared", "-fPIC", str(src), "-o", str(lib)], check=True)
    monkeypatch.setattr(cp, "_lib", None)
    monkeypatch.setattr(cp, "library_path", lambda: str(lib))
    with pytest.raises(cp.CoverPruneError, match=match):
        cp.uncovered_cost((1.0, 1.0, 1.0))
