"""Streams of rounds without end, one round at a time: what each layer keeps of the past is an 8-bit cache or a state.

A stream's rounds come one after the other, one token for each site.  Two layers look back over them:

    h += P_a(attention8(rope(q), cache))     the last rounds, kept as keys and values in 8 bits in a ring
    h += P_b(linear_attention(q, k, v))      all rounds, in a state of fixed size that fades with a slope for each head

Each layer's norm adds what the layer before left and gives the next product's codes and scales.

    python examples/stream_rounds.py [--d 13] [--rounds 50] [--kept 20] [--streams 4] [--codes e4m3|int8]

Random weights: it shows how the operators go together, and times a round.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_12841_amd as pdx  # noqa: E402

MOST = {"e4m3": (torch.float8_e4m3fn, 448.0), "int8": (torch.int8, 127.0)}


def quantise(w, codes):
    """Weights [N][K] as 8-bit codes with one scale an output channel."""
    dtype, most = MOST[codes]
    scale = w.abs().amax(1).clamp(min=1e-30) / most
    v = w / scale[:, None]
    return (v.round() if codes == "int8" else v).to(dtype), scale


class StreamLayers:
    """Weights, caches, states and buffers of the two layers for `streams` streams of rounds of (d + 1)^2 tokens; `kept` rounds in the ring."""

    def __init__(self, streams, d, kept, width=128, heads=4, kv_heads=2, codes="e4m3", cap=30.0, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.streams, self.grid, self.width, self.heads, self.kv_heads = streams, (d + 1) ** 2, width, heads, kv_heads
        self.head_dim, self.cap = width // heads, cap
        n, qkv = streams * self.grid, (heads + 2 * kv_heads) * self.head_dim

        def weights(rows, cols):
            return quantise(torch.randn(rows, cols, generator=g, device=device) / cols ** 0.5, codes)
        self.w = {name: weights(*shape) for name, shape in (("qkv", (qkv, width)), ("out", (width, width)), ("linear_qkv", (qkv, width)),
                                                            ("linear_out", (width, width)))}
        pairs = self.head_dim // 2
        self.sections = (pairs - 2 * (pairs // 4), pairs // 4, pairs // 4)
        self.slopes = torch.exp2(-8.0 * (torch.arange(heads, device=device) + 1.0) / heads)
        self.fades = torch.exp2(-6.0 * (torch.arange(kv_heads, device=device) + 1.0) / kv_heads)
        self.cache = pdx.new_cache(streams, kept * self.grid, kv_heads, self.head_dim, codes, device)
        self.at = torch.zeros(streams, dtype=torch.int64, device=device)  # the place of the next round in the ring
        self.state = torch.zeros(streams, kv_heads, self.head_dim, self.head_dim, device=device)
        bf = dict(dtype=torch.bfloat16, device=device)
        self.qkv, self.linear_qkv = torch.empty(n, qkv, **bf), torch.empty(n, qkv, **bf)
        self.seen, self.product, self.last = torch.empty(n, width, **bf), torch.empty(n, width, **bf), torch.empty(n, width, **bf)
        self.codes, self.scales = torch.empty(n, width, dtype=MOST[codes][0], device=device), torch.empty(n, device=device)

    def _parts(self, qkv):
        """Queries, keys and values [streams][tokens][heads][head_dim] in the rows of a joint projection."""
        return qkv.view(self.streams, self.grid, -1, self.head_dim).split([self.heads, self.kv_heads, self.kv_heads], 2)

    def run(self, h, sites):
        """A round of every stream: h [streams grid][width] (updated in place), sites [streams][grid][4].  Returns what is left to add."""
        H, Hk, D = self.heads, self.kv_heads, self.head_dim
        pdx.rms_norm(h, codes=self.codes, scales=self.scales)
        pdx.matmul8(self.codes, self.scales, *self.w["qkv"], self.qkv)
        turned = self.qkv.view(-1, H + 2 * Hk, D)[:, :H + Hk]
        pdx.rope(turned, sites.view(-1, 4), turned, self.sections, base=100.0)
        q, k, v = self._parts(self.qkv)
        pdx.cache_write(self.cache, self.at, k, v, sites)
        self.at += self.grid
        pdx.attention8(q, self.cache, self.seen.view(self.streams, self.grid, H, D), sites, cap=self.cap, slopes=self.slopes, causal=True)
        pdx.rms_norm(self.seen, codes=self.codes, scales=self.scales)
        pdx.matmul8(self.codes, self.scales, *self.w["out"], self.product)
        pdx.rms_norm(h, residual=self.product, sum_out=h, codes=self.codes, scales=self.scales)
        pdx.matmul8(self.codes, self.scales, *self.w["linear_qkv"], self.linear_qkv)
        q, k, v = self._parts(self.linear_qkv)
        pdx.linear_attention(q, k, v, self.seen.view(self.streams, self.grid, H, D), slopes=self.fades, per_round=self.grid, state=self.state,
                             state_out=self.state)
        pdx.rms_norm(self.seen, codes=self.codes, scales=self.scales)
        pdx.matmul8(self.codes, self.scales, *self.w["linear_out"], self.last)
        return self.last


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--d", type=int, default=13)
    p.add_argument("--rounds", type=int, default=50)
    p.add_argument("--kept", type=int, default=20)
    p.add_argument("--streams", type=int, default=4)
    p.add_argument("--codes", choices=sorted(MOST), default="e4m3")
    a = p.parse_args()
    layers = StreamLayers(a.streams, a.d, a.kept, codes=a.codes)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    site = pdx.volume_sites(a.d, 1)
    sites = site.repeat(a.streams, 1, 1)
    sites[..., 3] = torch.arange(a.streams, device="cuda", dtype=torch.int32)[:, None]
    h = torch.empty(a.streams * layers.grid, 128, dtype=torch.bfloat16, device="cuda")
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for t in range(a.rounds):
        h.normal_(generator=g)
        sites[..., 0] = t
        begin.record()
        left = layers.run(h, sites)
        end.record()
    h += left
    torch.cuda.synchronize()
    held = layers.cache[0].numel() + 4 * layers.cache[1].numel() + 4 * layers.cache[2].numel()
    print("%d streams of d = %d, %d rounds, %d kept: %.0f us for a round of all" % (a.streams, a.d, a.rounds, a.kept, begin.elapsed_time(end) * 1e3))
    print("%.1f kB of cache and %.1f kB of state a stream; rms of the residual stream %.3f" %
          (held / a.streams / 1e3, layers.state.numel() * 4 / a.streams / 1e3, h.float().square().mean().sqrt()))


if __name__ == "__main__":
    main()
