"""The example's decoder with a cache of 4 bits and with a budget: it runs, the cache is what it should be, and what attends to
it is what is in it."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("prune_then_decode", os.path.join(ROOT, "examples", "prune_then_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("budget", [0, 100])
def test_decoder(bits, budget):
    ex = _example()
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(300, 512, device="cuda", generator=g).to(torch.bfloat16)
    positions = (torch.arange(300, device="cuda") * 17 % 3001).sort().values.to(torch.int32)
    model, rows, _ = ex.run(x, positions, 70, 2, 8, 2, bits=bits, budget=budget)
    assert rows.shape == (70, 512) and bool(torch.isfinite(rows.float()).all())
    # The prompt leaves 100, 64 more tokens make it 100 again, six follow.
    assert model.length == (106 if budget else 370)
    assert model.cache_bytes() == 2 * 2 * model.length * 2 * (34 if bits == 4 else 128)
    for mass in model.mass:
        # A token has weight, nothing else does; each of a group's heads gives 1 at a time.
        assert bool((mass[:, :, model.length:] == 0).all()) and bool((mass[:, :, :model.length] > 0).all())


def test_a_budget_that_is_not_reached_changes_nothing():
    ex = _example()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(90, 512, device="cuda", generator=g).to(torch.bfloat16)
    positions = torch.arange(90, device="cuda", dtype=torch.int32)
    a, b = (ex.run(x, positions, 8, 2, 8, 2, bits=4, budget=n)[1] for n in (0, 5000))
    assert torch.equal(a, b)
