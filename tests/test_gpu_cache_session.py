"""The operators that keep a session's cache small, together: a prompt into a 4-bit cache, its last rows' attention adding up
masses, eviction, further tokens in the places that fell free; on other streams and in replayed graphs."""
import math

import pytest

from tests import cache_ref, serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def _same(xs, ys):
    """Bit for bit (unused slots hold NaN)."""
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(xs, ys, strict=True))


class _Session:
    """Sequences in a cache of `held`: appends, attends with masses, evicts."""

    def __init__(self, batch=2, held="e2m1", hq=8, hk=2, d=128, page=16, room=1200, seed=0):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.hq, self.hk, self.d, self.page, self.held, self.batch = hq, hk, d, page, held, batch
        width = (room + page - 1) // page
        self.room = width * page
        self.table = torch.randperm(batch * width, device="cuda", generator=self.g).view(batch, width).to(torch.int32)
        shape = (batch * width, hk, page)
        if held == "e2m1":
            self.caches = [torch.full((*shape, d // 2), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(2)]
            self.scales = [torch.full((*shape, d // 32), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
        else:
            self.caches = [torch.full((*shape, d), math.nan, dtype=BF, device="cuda") for _ in range(2)]
            if held == "e4m3":
                self.caches = [x.to(E4M3) for x in self.caches]
            self.scales = [torch.full((hk,), 0.02, device="cuda") if held == "e4m3" else None for _ in range(2)]
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.mass = torch.zeros(batch, hk, self.room, device="cuda")
        self.inv = 10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)
        self.position = 0

    def rows(self, tokens):
        """Queries, keys and values of `tokens` new tokens of each sequence."""
        x = torch.randn(self.batch * tokens, self.hq + 2 * self.hk, self.d, device="cuda", generator=self.g).to(BF)
        return x.split([self.hq, self.hk, self.hk], 1)

    def append(self, qkv, tokens):
        import paper_2608_13226_amd as cp
        at = self.lengths[:, None].long() + torch.arange(tokens, device="cuda")
        slots = (self.table.long().gather(1, at // self.page) * self.page + at % self.page).flatten()
        pos = (self.position + torch.arange(tokens, device="cuda", dtype=torch.int32)).repeat(self.batch)
        if self.held == "e2m1":
            q = cp.kv_append4(*qkv, pos, slots, self.inv, *self.caches, *self.scales)
        else:
            q = cp.kv_append(*qkv, pos, slots, self.inv, *self.caches, k_scale=self.scales[0], v_scale=self.scales[1])
        self.lengths += tokens
        return q, slots

    def attend(self, q, longest, **kw):
        import paper_2608_13226_amd as cp
        return cp.paged_attention_mass(q, *self.caches, self.table, self.lengths, self.mass, max_length=longest, k_scale=self.scales[0],
                                       v_scale=self.scales[1], **kw)

    def evict(self, keep, longest, **kw):
        import paper_2608_13226_amd as cp
        four = self.held == "e2m1"
        return cp.kv_evict(*self.caches, self.table, self.lengths, self.mass, keep, recent=32, sink=4, max_length=longest,
                           k_scale=self.scales[0] if four else None, v_scale=self.scales[1] if four else None, mass_out=self.mass, **kw)

    def read(self, i, n):
        """Sequence i's first n keys and values."""
        import paper_2608_13226_amd as cp
        at = torch.arange(n, device="cuda")
        return cp.kv_gather(*self.caches, self.table[i].long()[at // self.page] * self.page + at % self.page, BF, *self.scales)

    def expected(self, q):
        return cache_ref.attend(q, *self.caches, self.table, self.lengths, k_scale=self.scales[0], v_scale=self.scales[1])


def _near(got, want, size, tokens, d):
    # As in the attention's own tests: float32 work on scores below 60.
    ref.assert_close(got, want, got.dtype, 2.0 ** -24 * (60 * (d / 32 + 8) + tokens / 32 + 100) * size, "out")


@pytest.mark.parametrize("held", ["e2m1", "e4m3", "bf16"])
def test_a_session(held):
    s = _Session(held=held)
    qkv = s.rows(900)
    q, _ = s.append(qkv, 900)
    s.position = 900
    # The prompt's last rows, as sequences of their own over the same pages, say what counts.
    import paper_2608_13226_amd as cp
    last = q.view(s.batch, 900, s.hq, s.d)[:, -16:].flatten(0, 1).contiguous()
    lengths = (torch.arange(885, 901, device="cuda", dtype=torch.int32)).repeat(s.batch)
    mass = torch.zeros(16 * s.batch, s.hk, s.room, device="cuda")
    cp.paged_attention_mass(last, *s.caches, s.table.repeat_interleave(16, 0).contiguous(), lengths, mass, max_length=900, k_scale=s.scales[0],
                            v_scale=s.scales[1])
    want = cache_ref.attend(last, *s.caches, s.table.repeat_interleave(16, 0), lengths, k_scale=s.scales[0], v_scale=s.scales[1])[3]
    s.mass += mass.view(s.batch, 16, s.hk, s.room).sum(1)
    assert bool(((s.mass[:, :, :900].cpu() - want.view(s.batch, 16, s.hk, 900).sum(1)).abs() < 1e-4).all())

    before = [s.read(i, 900) for i in range(s.batch)]
    r = s.evict(300, 900)
    s.lengths = r.lengths
    assert r.lengths.tolist() == [300] * s.batch
    for i in range(s.batch):
        for x, y in zip(s.read(i, 300), before[i]):
            assert torch.equal(x, torch.stack([y[r.kept[i, h].long(), h] for h in range(s.hk)], 1))
        assert torch.equal(r.kept[i, :, -32:], torch.arange(868, 900, device="cuda", dtype=torch.int32).expand(s.hk, 32))
        assert bool((r.kept[i, :, :4] == torch.arange(4, device="cuda", dtype=torch.int32)).all())

    # Decoded tokens follow in the places that fell free; old rows there are not seen.
    for step in range(6):
        q, _ = s.append(s.rows(1), 1)
        s.position += 1
        out = s.attend(q, 320)
        want, _, size, _ = s.expected(q)
        _near(out, want, size, 310, s.d)
    assert bool((s.mass[:, :, 306:] == 0).all()) and bool((s.mass[:, :, :306] > 0).all())
    # Down to the budget again.
    r = s.evict(300, 320)
    s.lengths = r.lengths
    q, _ = s.append(s.rows(1), 1)
    out = s.attend(q, 320)
    want, _, size, _ = s.expected(q)
    _near(out, want, size, 310, s.d)


class _Step:
    """One decode step that drops a token: append at fixed slots, attention with masses, eviction."""

    def __init__(self, long=False, held="e2m1", seed=0):
        room = 20000 if long else 700
        self.s = _Session(batch=3, held=held, room=room, seed=seed)
        n = room - 20
        self.keep, self.longest = (n // 2, n) if long else (n - 40, n)
        self.s.append(self.s.rows(n - 1), n - 1)
        self.s.position = n - 1
        self.s.mass.copy_(torch.rand(self.s.mass.shape, device="cuda", generator=self.s.g))
        self.s.lengths += 1
        at = self.s.lengths.long() - 1
        self.slots = self.s.table.long().gather(1, (at // 16)[:, None])[:, 0] * 16 + at % 16
        self.pos = torch.full((3,), n, dtype=torch.int32, device="cuda")
        self.qkv = self.s.rows(1)

    def state(self):
        return [*self.s.caches, *[x for x in self.s.scales if x is not None], self.s.mass]

    def __call__(self):
        import paper_2608_13226_amd as cp
        s = self.s
        if s.held == "e2m1":
            q = cp.kv_append4(*self.qkv, self.pos, self.slots, s.inv, *s.caches, *s.scales)
            a = cp.paged_attention4(q, *s.caches, *s.scales, s.table, s.lengths, max_length=self.longest)
        else:
            q = cp.kv_append(*self.qkv, self.pos, self.slots, s.inv, *s.caches)
            a = cp.paged_attention(q, *s.caches, s.table, s.lengths, max_length=self.longest)
        o = s.attend(q, self.longest)
        r = s.evict(self.keep, self.longest)
        return [q, a, o, r.kept, r.lengths, r.mass, *cp.kv_gather(*s.caches, self.slots, BF, *s.scales)]


@pytest.mark.parametrize("long", [False, True])
def test_on_another_stream(long):
    a, b = _Step(long), _Step(long)
    want = a()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = b()
    s.synchronize()
    assert _same([*got, *b.state()], [*want, *a.state()])


@pytest.mark.parametrize("long", [False, True])
def test_the_stream_argument(long):
    import paper_2608_13226_amd as cp
    a = _Step(long)
    s = torch.cuda.Stream()
    # (The sequences' last token, whose blocks are NaN until then.)
    cp.kv_append4(*a.qkv, a.pos, a.slots, a.s.inv, *a.s.caches, *a.s.scales)
    want = cp.paged_attention4(a.qkv[0].contiguous(), *a.s.caches, *a.s.scales, a.s.table, a.s.lengths, max_length=a.longest)
    s.wait_stream(torch.cuda.current_stream())
    got = cp.paged_attention4(a.qkv[0].contiguous(), *a.s.caches, *a.s.scales, a.s.table, a.s.lengths, max_length=a.longest, stream=s)
    k, v = cp.kv_gather(*a.s.caches, a.slots, BF, *a.s.scales, stream=s)
    r = cp.kv_evict(*a.s.caches, a.s.table, a.s.lengths, a.s.mass, a.keep, max_length=a.longest, k_scale=a.s.scales[0],
                    v_scale=a.s.scales[1], stream=s)
    s.synchronize()
    assert torch.equal(got, want) and k.shape == v.shape and r.lengths.tolist() == [a.keep] * 3


@pytest.mark.parametrize("held", ["e2m1", "bf16"])
@pytest.mark.parametrize("long", [False, True])
def test_in_a_graph(long, held):
    step, eager = _Step(long, held), _Step(long, held)
    s = torch.cuda.Stream()
    start = [x.clone() for x in step.state()]
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for x, y in zip(step.state(), start):
        x.copy_(y)
    for i in range(4):
        # New inputs in place, eager work and a synchronization between the replays; the cache goes on changing.
        for a in (step, eager):
            g = torch.Generator(device="cuda").manual_seed(100 + i)
            for x in a.qkv:
                x.copy_(torch.randn(x.shape, device="cuda", generator=g))
            a.s.mass.add_(torch.rand(a.s.mass.shape, device="cuda", generator=g))
            a.pos.add_(3)
        graph.replay()
        torch.cuda.synchronize()
        want = eager()
        torch.cuda.synchronize()
        assert _same(out, want), f"replay {i}"
        assert _same(step.state(), eager.state()), f"state after replay {i}"


def test_two_graphs_with_one_workspace():
    """Replayed one after another, as calls on one stream are."""
    import paper_2608_13226_amd as cp
    lib = cp.library()
    steps = [_Step(True, seed=i) for i in range(2)]
    a = steps[0]
    bytes_ = max(lib.coverprune_paged_attention_mass_workspace(3, 8, 2, 128, a.longest, 0),
                 lib.coverprune_kv_evict_workspace(3, 2, a.keep, 32, a.longest))
    ws = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
    wants, graphs, outs = [], [], []

    def run(step):
        q = step.qkv[0].contiguous()
        o = step.s.attend(q, step.longest, workspace=ws)
        r = step.s.evict(step.keep, step.longest, workspace=ws)
        return [o, *r]

    for i, step in enumerate(steps):
        other = _Step(True, seed=i)
        wants.append([[x.clone() for x in run(other)] for _ in range(2)])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(run(step))
        graphs.append(graph)
    for n in range(2):
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert _same(outs[i], wants[i][n]), f"graph {i}, replay {n}"


def test_two_streams_at_once():
    steps, others = [_Step(True, seed=i) for i in range(2)], [_Step(True, seed=i) for i in range(2)]
    wants = [x() for x in others]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    gots = []
    for step, s in zip(steps, streams):
        with torch.cuda.stream(s):
            gots.append(step())
    torch.cuda.synchronize()
    for got, want, a, b in zip(gots, wants, steps, others):
        assert _same([*got, *a.state()], [*want, *b.state()])


def _calls(step):
    import paper_2608_13226_amd as cp
    s = step.s
    q = step.qkv[0].contiguous()
    q2, o, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(3, s.hq, device="cuda")
    ws = torch.empty(1 << 24, device="cuda", dtype=torch.uint8)
    k, v = (torch.empty(3, s.hk, s.d, dtype=BF, device="cuda") for _ in range(2))
    kept = torch.empty(3, s.hk, step.keep, dtype=torch.int32, device="cuda")
    left, now = torch.empty_like(s.mass), torch.empty_like(s.lengths)
    scales = dict(k_scale=s.scales[0], v_scale=s.scales[1])
    return [
        (lambda: cp.kv_append4(*step.qkv, step.pos, step.slots, s.inv, *s.caches, *s.scales, q_out=q2), [*s.caches, *s.scales, q2]),
        (lambda: cp.kv_gather(*s.caches, step.slots, BF, *s.scales, k_out=k, v_out=v), [k, v]),
        (lambda: cp.paged_attention4(q, *s.caches, *s.scales, s.table, s.lengths, max_length=step.longest, out=o, lse=lse, workspace=ws), [o, lse, ws]),
        (lambda: cp.paged_attention_mass(q, *s.caches, s.table, s.lengths, s.mass, max_length=step.longest, **scales, out=o, lse=lse,
                                         workspace=ws), [o, lse, s.mass, ws]),
        (lambda: cp.kv_evict(*s.caches, s.table, s.lengths, s.mass, step.keep, max_length=step.longest, **scales, kept=kept, mass_out=left,
                             lengths_out=now, workspace=ws), [*s.caches, *s.scales, kept, left, now, ws])]


def test_autograd_knows_what_was_written():
    for call, outputs in _calls(_Step()):
        before = [t._version for t in outputs]
        call()
        assert all(t._version > v for t, v in zip(outputs, before))


def test_tensors_of_another_gpu_than_the_current_one():
    """Refused by each operator: the library launches on the current GPU.  (One GPU is enough: the binding is told
    that another is current.)"""
    import paper_2608_13226_amd as cp
    from paper_2608_13226_amd import serving
    step = _Step()
    step()
    before = [x.clone() for x in step.state()]
    serving._native.init(cp.CoverPruneError, serving._raw_stream, lambda: torch.cuda.current_device() + 1)
    try:
        for call, _ in _calls(step):
            with pytest.raises(ValueError, match="current GPU"):
                call()
    finally:
        serving._native.init(cp.CoverPruneError, serving._raw_stream, serving._device)
    assert _same(step.state(), before)
