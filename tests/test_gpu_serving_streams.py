"""The serving operators on a stream of their own and in a replayed graph: one
decode step, norm -> product -> append -> attention -> product."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF = torch.bfloat16


class _Step:
    def __init__(self, batch=3, length=900, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.hq, self.hk, self.d, self.page = 8, 2, 128, 16
        dim, width = self.hq * self.d, (length + 15) // 16 + 1

        def w4(n, k):
            return (torch.randint(0, 256, (n, k // 2), device="cuda", generator=g, dtype=torch.uint8),
                    (0.01 + 0.01 * torch.rand(n, k // 128, device="cuda", generator=g)).to(BF))

        self.x = torch.randn(batch, dim, device="cuda", generator=g).to(BF)
        self.h = torch.randn(batch, dim, device="cuda", generator=g).to(BF)
        self.gain = torch.ones(dim, device="cuda", dtype=BF)
        self.wqkv, self.wo = w4((self.hq + 2 * self.hk) * self.d, dim), w4(dim, dim)
        self.k, self.v = (torch.randn(batch * width, self.hk, 16, self.d, device="cuda", generator=g).to(BF) for _ in range(2))
        self.table = torch.arange(batch * width, device="cuda", dtype=torch.int32).view(batch, width)
        self.lengths = torch.full((batch,), length, device="cuda", dtype=torch.int32)
        self.positions = self.lengths * 7
        at = self.lengths.long() - 1
        self.slots = self.table.long().gather(1, (at // 16)[:, None])[:, 0] * 16 + at % 16
        self.inv = 10000.0 ** (-torch.arange(0, self.d, 2, device="cuda") / self.d)
        self.length = length

    def __call__(self):
        import paper_2608_13226_amd as cp
        r = cp.rms_norm(self.x, self.gain, residual=self.h, quantize=True)
        qkv = cp.w4_matvec(r.out, *self.wqkv, x_scale=r.scale).unflatten(1, (-1, self.d))
        q, k, v = qkv.split([self.hq, self.hk, self.hk], 1)
        q = cp.kv_append(q, k, v, self.positions, self.slots, self.inv, self.k, self.v)
        o = cp.paged_attention(q, self.k, self.v, self.table, self.lengths, max_length=self.length)
        return cp.w4_matvec(o.flatten(1), *self.wo), r.residual


def test_on_another_stream():
    step = _Step()
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = step()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("length", [900, 20000])
def test_in_a_graph(length):
    step = _Step(length=length)
    step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        # New inputs in place, eager work and a synchronization between the replays.
        g = torch.Generator(device="cuda").manual_seed(100 + i)
        step.x.copy_(torch.randn(step.x.shape, device="cuda", generator=g))
        step.positions.add_(3)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), f"replay {i}"


def test_tensors_of_another_gpu_than_the_current_one():
    """Refused by each operator: the library launches on the current GPU.  (One GPU is enough: the binding is told
    that another is current.)"""
    import paper_2608_13226_amd as cp
    from paper_2608_13226_amd import serving
    step = _Step()
    want = [t.clone() for t in step()]
    q = torch.zeros(3, 8, 128, device="cuda", dtype=BF)
    calls = [lambda: cp.rms_norm(step.x, step.gain), lambda: cp.w4_matvec(step.x, *step.wo),
             lambda: cp.kv_append(q, q[:, :2], q[:, :2], step.positions, step.slots, step.inv, step.k, step.v),
             lambda: cp.paged_attention(q, step.k, step.v, step.table, step.lengths)]
    serving._native.init(cp.CoverPruneError, serving._raw_stream, lambda: torch.cuda.current_device() + 1)
    try:
        for call in calls:
            with pytest.raises(ValueError, match="current GPU"):
                call()
    finally:
        serving._native.init(cp.CoverPruneError, serving._raw_stream, serving._device)
    assert all(torch.equal(a, b) for a, b in zip(step(), want))


def test_autograd_knows_what_was_written():
    """A tensor that an operator writes counts as modified in place, so that a backward pass through its old values raises."""
    import paper_2608_13226_amd as cp
    step = _Step()
    q = torch.zeros(3, 8, 128, device="cuda", dtype=BF)
    k = torch.zeros(3, 2, 128, device="cuda", dtype=BF)
    out, y, lse = torch.empty_like(step.x), torch.empty_like(step.x), torch.empty(3, 8, device="cuda")
    codes = torch.empty(step.x.shape, device="cuda", dtype=torch.float8_e4m3fn)
    scale, r = torch.empty(3, device="cuda"), step.h.clone()
    o, q2 = torch.empty_like(q), torch.empty_like(q)
    ws = torch.empty(1 << 22, device="cuda", dtype=torch.uint8)
    calls = [(lambda: cp.rms_norm(step.x, step.gain, residual=r, residual_out=r, out=out), [out, r]),
             (lambda: cp.rms_norm(step.x, step.gain, quantize=True, out=codes, out_scale=scale), [codes, scale]),
             (lambda: cp.w4_matvec(step.x, *step.wo, out=y), [y]),
             (lambda: cp.kv_append(q, k, k, step.positions, step.slots, step.inv, step.k, step.v, q_out=q2), [step.k, step.v, q2]),
             (lambda: cp.paged_attention(q, step.k, step.v, step.table, step.lengths, out=o, lse=lse, workspace=ws), [o, lse, ws])]
    for call, outputs in calls:
        before = [t._version for t in outputs]
        call()
        assert all(t._version > v for t, v in zip(outputs, before))
    w = torch.ones_like(step.k, requires_grad=True)
    loss = (w * step.k).float().sum()
    cp.kv_append(q, k, k, step.positions, step.slots, step.inv, step.k, step.v)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    with torch.inference_mode():
        cache = torch.zeros_like(step.k)
        cp.kv_append(None, k, k, step.positions, step.slots, step.inv, cache, torch.zeros_like(cache))
