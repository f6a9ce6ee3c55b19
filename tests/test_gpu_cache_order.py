"""A session's operators on a stream of their own, and captured and replayed, where the stream waits for what the default
one has still under way: the caches' filling, the copies of their state and of the arguments."""
import pytest

from tests.test_gpu_cache_session import BF, _same, _Step

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("held", ["e2m1", "bf16"])
@pytest.mark.parametrize("long", [False, True])
def test_a_replayed_step(long, held):
    step, eager = _Step(long, held), _Step(long, held)
    start = [x.clone() for x in step.state()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    for x, y in zip(step.state(), start):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    # A capture runs nothing.
    assert _same(step.state(), start) and _same(eager.state(), start)
    for i in range(4):
        for a in (step, eager):
            g = torch.Generator(device="cuda").manual_seed(200 + i)
            for x in a.qkv:
                x.copy_(torch.randn(x.shape, device="cuda", generator=g))
            a.s.mass.add_(torch.rand(a.s.mass.shape, device="cuda", generator=g))
            a.pos.add_(5)
        graph.replay()
        want = eager()
        torch.cuda.synchronize()
        assert _same(out, want), f"replay {i}"
        assert _same(step.state(), eager.state()), f"state after replay {i}"


@pytest.mark.parametrize("long", [False, True])
def test_the_stream_argument_after_a_wait(long):
    """Every operator's, one after another on the stream that each is given."""
    import paper_2608_13226_amd as cp
    a, b = _Step(long), _Step(long)
    want = a()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    t = b.s
    q2 = cp.kv_append4(*b.qkv, b.pos, b.slots, t.inv, *t.caches, *t.scales, stream=s)
    o4 = cp.paged_attention4(q2, *t.caches, *t.scales, t.table, t.lengths, max_length=b.longest, stream=s)
    o = cp.paged_attention_mass(q2, *t.caches, t.table, t.lengths, t.mass, max_length=b.longest, k_scale=t.scales[0], v_scale=t.scales[1],
                                stream=s)
    r = cp.kv_evict(*t.caches, t.table, t.lengths, t.mass, b.keep, recent=32, sink=4, max_length=b.longest, k_scale=t.scales[0],
                    v_scale=t.scales[1], mass_out=t.mass, stream=s)
    k, v = cp.kv_gather(*t.caches, b.slots, BF, *t.scales, stream=s)
    s.synchronize()
    assert _same([q2, o4, o, r.kept, r.lengths, r.mass, k, v], want) and _same(b.state(), a.state())
