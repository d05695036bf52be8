"""A block of attention over the sites of detector volumes, behind the conv layers of the pre-decoder.

The pre-decoder's networks see their receptive field.  This example takes the activations of one of its
layers as tokens, one for each site of each round, and runs a block over whole volumes with the token operators, the products
in 8 bits:

    h += P_out(norm(attention(rope(P_qkv(norm(h))))))
    h += P_down(norm(gelu(P_up(norm(h)))))

Every norm also adds the product before it to the residual stream h and gives the next product's codes and scales.

    python examples/volume_block.py [--d 13] [--T 13] [--batch 16] [--codes e4m3|int8] [--causal]

Random weights: it shows how the operators go together, and times them.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_12841_amd as pdx  # noqa: E402
from paper_2604_12841_amd import workload  # noqa: E402

CODES = {"e4m3": (torch.float8_e4m3fn, 448.0), "int8": (torch.int8, 127.0)}


def quantise(w, codes):
    """Weights [N][K] as 8-bit codes with one scale an output channel."""
    dtype, most = CODES[codes]
    scale = w.abs().amax(1).clamp(min=1e-30) / most
    v = w / scale[:, None]
    return (v.round() if codes == "int8" else v).to(dtype), scale


class VolumeBlock:
    """Weights and buffers of one block for `tokens` tokens of `width` channels."""

    def __init__(self, tokens, width=128, heads=8, kv_heads=2, hidden=512, codes="e4m3", cap=30.0, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.width, self.heads, self.kv_heads, self.head_dim = width, heads, kv_heads, width // heads
        self.cap, dtype = cap, CODES[codes][0]
        qkv = (heads + 2 * kv_heads) * self.head_dim

        def weights(n, k):
            return quantise(torch.randn(n, k, generator=g, device=device) / k ** 0.5, codes)
        self.w_qkv, self.w_out, self.w_up, self.w_down = weights(qkv, width), weights(width, width), weights(hidden, width), weights(width, hidden)
        self.gains = [torch.ones(n, device=device) for n in (width, width, width, hidden)]
        pairs = self.head_dim // 2
        self.sections = (pairs - 2 * (pairs // 4), pairs // 4, pairs // 4)
        # heads look near to far: one slope each
        self.slopes = torch.exp2(-8.0 * (torch.arange(heads, device=device) + 1.0) / heads)
        bf = dict(dtype=torch.bfloat16, device=device)
        self.qkv, self.attended = torch.empty(tokens, qkv, **bf), torch.empty(tokens, width, **bf)
        self.product, self.hidden = torch.empty(tokens, width, **bf), torch.empty(tokens, hidden, **bf)
        self.codes = torch.empty(tokens, width, dtype=dtype, device=device)
        self.hidden_codes = torch.empty(tokens, hidden, dtype=dtype, device=device)
        self.scales = torch.empty(tokens, device=device)

    def run(self, h, sites, batch, added=None, causal=False):
        """h [tokens][width] (the residual stream, updated in place), plus `added` if given (what the block before left
        to add).  Returns this block's last product, which the next norm adds.  sites [tokens / batch][4] or [batch][..][4]."""
        n, H, Hk, D = h.shape[0], self.heads, self.kv_heads, self.head_dim
        pdx.rms_norm(h, self.gains[0], residual=added, sum_out=h if added is not None else None, codes=self.codes, scales=self.scales)
        pdx.matmul8(self.codes, self.scales, *self.w_qkv, self.qkv)
        qkv = self.qkv.view(n, H + 2 * Hk, D)
        flat = sites if sites.dim() == 2 and batch == 1 else sites.expand(batch, n // batch, 4).reshape(n, 4)
        pdx.rope(qkv[:, :H + Hk], flat, qkv[:, :H + Hk], self.sections, base=100.0)
        q, k, v = qkv.view(batch, n // batch, H + 2 * Hk, D).split([H, Hk, Hk], 2)
        pdx.attention(q, k, v, self.attended.view(batch, n // batch, H, D), sites, sites, cap=self.cap, slopes=self.slopes, causal=causal)
        pdx.rms_norm(self.attended, self.gains[1], codes=self.codes, scales=self.scales)
        pdx.matmul8(self.codes, self.scales, *self.w_out, self.product)
        pdx.rms_norm(h, self.gains[2], residual=self.product, sum_out=h, codes=self.codes, scales=self.scales)
        pdx.matmul8(self.codes, self.scales, *self.w_up, self.hidden, act="gelu")
        pdx.rms_norm(self.hidden, self.gains[3], codes=self.hidden_codes, scales=self.scales)
        pdx.matmul8(self.hidden_codes, self.scales, *self.w_down, self.product)
        return self.product


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--d", type=int, default=13)
    p.add_argument("--T", type=int, default=13)
    p.add_argument("--batch", type=int, default=16)
    p.add_argument("--codes", choices=sorted(CODES), default="e4m3")
    p.add_argument("--causal", action="store_true")
    a = p.parse_args()
    layers = workload.layer_spec(4, 128)
    pre = pdx.Predecoder(workload.he_normal_weights(layers, seed=1), a.d, a.T, layers, "bf16", max_batch=a.batch)
    det, _ = workload.make_inputs(a.d, a.T, a.batch, 0.005, 0.005, seed=2)
    det = torch.from_numpy(det.view("int64")).cuda()
    sites = pdx.volume_sites(a.d, a.T)
    tokens = a.batch * sites.shape[0]
    h = torch.empty(tokens, 128, dtype=torch.bfloat16, device="cuda")
    pre.activations(det, 2, h)  # the third hidden layer: [batch][T][d + 1][d + 1][128]
    block = VolumeBlock(tokens, codes=a.codes)
    start = h.clone()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for n in range(6):  # the first passes warm up
        h.copy_(start)
        begin.record()
        left = block.run(h, sites, a.batch, causal=a.causal)
        end.record()
    h += left
    torch.cuda.synchronize()
    print("%d volumes of d = %d, T = %d: %d tokens, %s codes, %.0f us a block" % (a.batch, a.d, a.T, tokens, a.codes, begin.elapsed_time(end) * 1e3))
    print("rms of the residual stream: %.3f before, %.3f after" % (start.float().square().mean().sqrt(), h.float().square().mean().sqrt()))


if __name__ == "__main__":
    main()
