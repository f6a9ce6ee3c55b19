"""The example that prunes a scene and decodes over the kept tokens: its
decoder against plain float32 arithmetic with the same 4-bit weights, and the
prefill against the same tokens one at a time."""
import importlib.util
import math
import os

import pytest

from tests import serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("prune_then_decode", os.path.join(ROOT, "examples", "prune_then_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _plain(model, x, positions):
    """The decoder's last rows in float64, every rounding left out."""
    hq, hk, d = model.heads, model.kv_heads, model.d
    lin = lambda x, w: x @ ref.unpack_w4(*w)[0].t()       # noqa: E731
    norm = lambda h, w: h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * ref.d64(w)   # noqa: E731
    n = x.shape[0]
    h = ref.d64(x)
    seen = torch.ones(n, n).tril().bool()
    for layer in model.layers:
        qkv = lin(norm(h, layer["norm1"]), layer["qkv"]).view(n, hq + 2 * hk, d)
        q, _ = ref.rotate(qkv[:, :hq], positions, model.inv_freq.cpu(), False, 1.0)
        k, _ = ref.rotate(qkv[:, hq:hq + hk], positions, model.inv_freq.cpu(), False, 1.0)
        v = qkv[:, hq + hk:]
        out = torch.zeros(n, hq, d, dtype=torch.float64)
        for i in range(hq):
            s = (q[:, i] @ k[:, i // (hq // hk)].t()) / math.sqrt(d)
            out[:, i] = torch.softmax(torch.where(seen, s, -math.inf), 1) @ v[:, i // (hq // hk)]
        h = h + lin(out.flatten(1), layer["out"])
        gate, up = lin(norm(h, layer["norm2"]), layer["up"]).chunk(2, 1)
        h = h + lin(gate * torch.sigmoid(gate) * up, layer["down"])
    return norm(h, model.norm)


def test_decoder_against_plain_arithmetic():
    ex = _example()
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(90, 512, device="cuda", generator=g).to(torch.bfloat16)
    positions = (torch.arange(90, device="cuda") * 17 % 1000).sort().values.to(torch.int32)
    model = ex.Decoder(512, 2, 8, 2, 90, seed=1)
    got = ref.d64(model.forward(x, positions))
    want = _plain(model, x, positions)
    # 8-bit rows before three of each layer's four products: errors of 2^-4 / sqrt(3) of each
    # element, at random, which a product of many leaves as that share of its result.
    err = float((got - want).norm() / want.norm())
    assert err < 4 * 2.0 ** -4 / math.sqrt(3), err


def test_prefill_is_the_same_as_one_at_a_time():
    ex = _example()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(40, 256, device="cuda", generator=g).to(torch.bfloat16)
    positions = torch.arange(40, device="cuda", dtype=torch.int32) * 3
    whole = ex.Decoder(256, 2, 4, 2, 40, page=16, seed=4)
    single = ex.Decoder(256, 2, 4, 2, 40, page=16, seed=4)
    a = whole.forward(x, positions)
    b = torch.cat([single.forward(x[i:i + 1], positions[i:i + 1]) for i in range(40)])
    # The same sums cut otherwise: a rounding of an intermediate row may differ and pass through 8 bits.
    assert float((a.float() - b.float()).norm() / a.float().norm()) < 2.0 ** -4
    assert whole.length == single.length == 40


def test_the_whole_example():
    import paper_2608_13226_amd as cp
    from scenes import make_scene, subscene, to_device
    import numpy as np
    ex = _example()
    s = make_scene("n4096_d1152", 0)
    s = subscene(s, np.sort(np.random.default_rng(0).choice(s.n, 384, replace=False)))
    t = to_device(s, "cuda:0")
    kept = cp.prune(t["feats"], t["pos"], t["frame"], t["capacity"], 38)[2].check().selected.long().sort().values
    x = (t["feats"].to(torch.bfloat16).float() * math.sqrt(1152)).to(torch.bfloat16)
    model, rows, ms = ex.run(x[kept].contiguous(), kept.to(torch.int32), 3, 1, 18, 3)
    assert model.length == 41 and rows.shape == (3, 1152) and bool(torch.isfinite(rows.float()).all()) and ms > 0
