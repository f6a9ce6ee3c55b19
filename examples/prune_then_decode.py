"""Prune a scene, then decode over the kept tokens.

A synthetic scene's visual tokens are pruned; the kept ones, in their order in
the video and at the positions they had there, go through a small random-init
decoder with 4-bit weights and a paged cache, and a few tokens are decoded
after them.  The same is done without the prune, and the time of a decode step
and the cache's size are printed for both.  The cache can be held in 4 bits, and
kept at a budget: where it has grown 64 tokens past it, the tokens of each head
that attention has given the least weight leave.

    python examples/prune_then_decode.py [--scene n4096_d1152] [--keep 0.1] [--layers 2] [--steps 16] [--bits 4] [--budget 512]

Everything on the path is a call of this library, but for the gated unit's
elementwise product.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2608_13226_amd as cp  # noqa: E402

BF16 = torch.bfloat16


def quantize_w4(w: torch.Tensor, group: int = 128):
    """[n, k] weights to 4-bit codes (two a byte, the even k low), scales and
    zero points of groups along k, rounded to nearest between each group's ends."""
    n, k = w.shape
    g = w.float().view(n, k // group, group)
    low, high = g.amin(2).clamp(max=0.0), g.amax(2).clamp(min=0.0)
    scale = ((high - low) / 15.0).clamp(min=1e-8).to(BF16)
    zero = (-low / scale.float()).round().clamp(0, 15)
    codes = (g / scale.float()[:, :, None] + zero[:, :, None]).round().clamp(0, 15).to(torch.uint8).view(n, k)
    return codes[:, 0::2] | codes[:, 1::2] << 4, scale, zero.to(torch.uint8)


class Decoder:
    """Layers of (norm, projections, rotation and append, attention, output
    projection, norm, gated unit) with one paged cache a layer, of 16 or 4 bits
    an element.  With a budget, each layer's tokens gather the weight that its
    last prompt rows and decoded tokens give them."""

    SLACK, VOTERS = 64, 32          # tokens past the budget before an eviction; prompt rows whose attention counts

    def __init__(self, dim, layers, heads, kv_heads, capacity, page=64, hidden=None, seed=0, device="cuda", bits=16, budget=0):
        self.dim, self.heads, self.kv_heads, self.d, self.page = dim, heads, kv_heads, dim // heads, page
        hidden = 2 * dim if hidden is None else hidden
        g = torch.Generator(device=device).manual_seed(seed)

        def w4(n, k):
            return quantize_w4(torch.randn(n, k, device=device, generator=g) / math.sqrt(k))

        self.layers = [dict(norm1=torch.ones(dim, device=device, dtype=BF16), norm2=torch.ones(dim, device=device, dtype=BF16),
                            qkv=w4((heads + 2 * kv_heads) * self.d, dim), out=w4(dim, heads * self.d),
                            up=w4(2 * hidden, dim), down=w4(dim, hidden)) for _ in range(layers)]
        self.norm = torch.ones(dim, device=device, dtype=BF16)
        self.inv_freq = 10000.0 ** (-torch.arange(0, self.d, 2, device=device) / self.d)
        pages = (capacity + page - 1) // page
        # Pages come from a pool in no particular order.
        self.table = torch.randperm(pages, device=device, generator=g).to(torch.int32)[None]
        self.bits, self.budget = bits, budget

        def cache(width, dtype):
            return [torch.zeros(pages, kv_heads, page, width, device=device, dtype=dtype) for _ in range(2)]

        self.cache = [cache(self.d // 2, torch.uint8) if bits == 4 else cache(self.d, BF16) for _ in range(layers)]
        self.scales = [cache(self.d // 32, torch.uint8) if bits == 4 else [None, None] for _ in range(layers)]
        self.mass = [torch.zeros(1, kv_heads, pages * page, device=device) for _ in range(layers if budget else 0)]
        self.length = 0

    def cache_bytes(self) -> int:
        row = self.d // 2 + self.d // 32 if self.bits == 4 else 2 * self.d
        return sum(2 * row * self.length * self.kv_heads for _ in self.layers)

    def _attend(self, i, q, table, lengths, longest):
        """Attention of layer i's rows; the weights of the last ones are added to its masses."""
        (k, v), (ks, vs) = self.cache[i], self.scales[i]
        if self.budget and q.shape[0] == 1:
            return cp.paged_attention_mass(q, k, v, table, lengths, self.mass[i], max_length=longest, k_scale=ks, v_scale=vs)
        if self.budget:
            last = q[-self.VOTERS:]
            mass = torch.zeros(last.shape[0], *self.mass[i].shape[1:], device=q.device)
            cp.paged_attention_mass(last, k, v, table[-self.VOTERS:], lengths[-self.VOTERS:], mass, max_length=longest, k_scale=ks, v_scale=vs)
            self.mass[i] += mass.sum(0, keepdim=True)
        if self.bits == 4:
            return cp.paged_attention4(q, k, v, ks, vs, table, lengths, max_length=longest)
        return cp.paged_attention(q, k, v, table, lengths, max_length=longest)

    def _evict(self):
        """Every layer's cache down to the budget; each head keeps its own tokens."""
        n = torch.full((1,), self.length, dtype=torch.int32, device=self.table.device)
        for (k, v), (ks, vs), mass in zip(self.cache, self.scales, self.mass):
            cp.kv_evict(k, v, self.table, n, mass, self.budget, recent=min(32, self.budget), max_length=self.length, k_scale=ks,
                        v_scale=vs, mass_out=mass)
        self.length = self.budget

    def _linear(self, x, scale, w):
        return cp.w4_matvec(x, w[0], w[1], zero=w[2], x_scale=scale)

    def forward(self, x: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
        """Rows x [tokens, dim] follow what the cache holds; positions [tokens]
        int32.  Returns the normed hidden rows.  Each row attends to the cache
        up to itself: a row is a sequence of its own length over one table."""
        tokens, first = x.shape[0], self.length
        at = torch.arange(first, first + tokens, device=x.device)
        slots = self.table[0, at // self.page].long() * self.page + at % self.page
        lengths = (at + 1).to(torch.int32)
        table = self.table.expand(tokens, -1).contiguous()
        h = None
        for i, layer in enumerate(self.layers):
            r = cp.rms_norm(x, layer["norm1"], residual=h, quantize=True)
            h = x if h is None else r.residual
            qkv = self._linear(r.out, r.scale, layer["qkv"]).unflatten(1, (-1, self.d))
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
            append = cp.kv_append4 if self.bits == 4 else cp.kv_append
            q = append(q, k, v, positions, slots, self.inv_freq, *self.cache[i], *(self.scales[i] if self.bits == 4 else ()))
            o = self._attend(i, q, table, lengths, first + tokens)
            x = self._linear(o.flatten(1), None, layer["out"])
            r = cp.rms_norm(x, layer["norm2"], residual=h, quantize=True)
            h = r.residual
            gate, up = self._linear(r.out, r.scale, layer["up"]).chunk(2, 1)
            x = self._linear((torch.nn.functional.silu(gate) * up), None, layer["down"])
        self.length = first + tokens
        if self.budget and self.length >= self.budget + self.SLACK:
            self._evict()
        return cp.rms_norm(x, self.norm, residual=h).out


def run(feats, positions, steps, layers, heads, kv_heads, seed=0, bits=16, budget=0):
    """Prefill with `feats` and decode `steps` tokens, each the last hidden row
    fed back.  Returns the decoder, the rows and the milliseconds of a step."""
    model = Decoder(feats.shape[1], layers, heads, kv_heads, feats.shape[0] + steps, seed=seed, bits=bits, budget=budget)
    x = model.forward(feats, positions)[-1:]
    last = int(positions[-1])
    rows, times = [], []
    for i in range(steps):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        x = model.forward(x, torch.full((1,), last + 1 + i, dtype=torch.int32, device=x.device))
        b.record()
        b.synchronize()
        rows.append(x)
        times.append(a.elapsed_time(b))
    return model, torch.cat(rows), sorted(times)[len(times) // 2]


def main():
    from scenes import CONFIGS, make_scene, to_device

    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--scene", default="n4096_d1152", choices=sorted(CONFIGS))
    ap.add_argument("--keep", type=float, default=0.1)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--bits", type=int, default=16, choices=(16, 4))
    ap.add_argument("--budget", type=int, default=0, help="tokens that a head keeps (0: all)")
    a = ap.parse_args()
    t = to_device(make_scene(a.scene, 0), "cuda:0")
    feats = t["feats"].to(BF16)
    n, dim = feats.shape
    dim -= dim % 128                                # whole heads of 64 and groups of 128
    heads = dim // 64
    kv_heads = next(k for k in (4, 3, 2, 1) if heads % k == 0)
    x = (feats[:, :dim].float() * math.sqrt(dim)).to(BF16).contiguous()
    picks = cp.prune(t["feats"], t["pos"], t["frame"], t["capacity"], max(1, round(a.keep * n)))[2].check()
    kept = picks.selected.long().sort().values      # video order
    where = torch.arange(n, dtype=torch.int32, device=x.device)
    for name, rows in (("all", where.long()), ("kept", kept)):
        model, _, ms = run(x[rows].contiguous(), where[rows].contiguous(), a.steps, a.layers, heads, kv_heads, bits=a.bits,
                           budget=a.budget)
        print(f"{name:5s} {rows.numel():6d} tokens: cache {model.cache_bytes() / 2**20:8.1f} MiB, decode step {ms:.3f} ms", flush=True)


if __name__ == "__main__":
    main()
