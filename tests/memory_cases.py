"""Plain 64-bit forms of what a stream keeps (8-bit cache, linear attention's state), and bounds on what their kernels may differ by."""
import math

import torch

import paper_2604_12841_amd as pdx
import token_cases as tc
from token_cases import U16, U32

QMAX = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


# ---- cache ----


def quantise64(x, codes_type):
    """(codes as 64-bit values, fp32 scales) of the rows of x: x / scale rounded once, the scale rounded to fp32 before."""
    x = x.double()
    q = QMAX[codes_type]
    scale = (x.abs().amax(-1) / q).float()
    s = scale.double()[..., None]
    y = torch.where(s > 0, x / torch.where(s > 0, s, 1.0), 0.0)
    if codes_type == torch.int8:
        y = torch.round(y).clamp(-127, 127)
    else:
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        y = (torch.round(y / step) * step).clamp(-448, 448)
    odd = ~torch.isfinite(x).all(-1)
    return torch.where(odd[..., None], 0.0, y), torch.where(odd, math.nan, scale)


def places(at, n, capacity):
    return (at[:, None] + torch.arange(n, device=at.device)) % capacity


def by_token(cache):
    """Keys and values of a cache in 64 bits, [batch][capacity][kv_heads][head_dim]."""
    codes, scales, _ = cache
    x = codes.double() * scales.double()[..., None]
    return x[:, 0].transpose(1, 2), x[:, 1].transpose(1, 2)


def filled_cache(g, B, capacity, Hk, D, codes, sites):
    """A cache whose places with a token hold random rows, and the others anything but E4M3's NaN in codes of tokens: here NaN
    scales and every code."""
    x = tc.normal(g, B, 2, Hk, capacity, D) * torch.exp(0.7 * tc.normal(g, B, 2, Hk, capacity, 1))
    y, scale = quantise64(x, CODES[codes])
    cache = pdx.new_cache(B, capacity, Hk, D, codes)
    cache[0].copy_(y.float().to(CODES[codes]))
    cache[1].copy_(scale)
    cache[2].copy_(sites)
    empty = (cache[2][..., 3] < 0)[:, None, None, :].expand(B, 2, Hk, capacity)
    cache[0].view(torch.uint8)[empty] = 0x7f if codes == "e4m3" else 0x80
    cache[1][empty] = math.nan
    return cache


def attention8_reference(q, cache, q_sites, scale, cap, slopes, causal, prefix):
    """(out, bound) in 64 bits: attention's definition over code scale."""
    k, v = by_token(cache)
    there = (cache[2][..., 3] >= 0)[..., None, None]
    k, v = torch.where(there, k, 0.0), torch.where(there, v, 0.0)
    want, moved, score = tc.attention64(q, k, v, q_sites, cache[2], scale, cap, slopes, causal, prefix)
    # a key's scale multiplies the score (one rounding more), the cap is met within 2^-20 of itself
    score += 2.0 ** -20 * cap + 4 * U32 * float((q.double().abs().amax() * k.abs().nan_to_num(0, 0, 0).amax()) * q.shape[-1] * abs(scale))
    return want, tc.attention_tolerance(want, moved, score)


# ---- linear attention ----


def linear64(q, k, v, slopes, per_round, lengths, state, scale):
    """(out, state, sizes of both: the same sums of absolute values, rounds of each entry) round by round in 64 bits; out is 0 behind an
    entry's length."""
    B, n, H, D = q.shape
    Hk = k.shape[2]
    out = torch.zeros(B, n, H, D, device=q.device, dtype=torch.float64)
    out_size = torch.zeros_like(out)
    S = torch.zeros(B, Hk, D, D, device=q.device, dtype=torch.float64)
    size, rounds = torch.zeros_like(S), []
    for b in range(B):
        m = n if lengths is None else min(max(int(lengths[b]), 0), n)
        for h in range(Hk):
            s = torch.zeros(D, D, device=q.device, dtype=torch.float64) if state is None else state[b, h].double()
            a = s.abs()
            fade = 1.0 if slopes is None else math.exp(-float(slopes[h]))
            qs = slice(h * (H // Hk), (h + 1) * (H // Hk))
            for lo in range(0, m, per_round):
                hi = min(m, lo + per_round)
                kk, vv = k[b, lo:hi, h].double(), v[b, lo:hi, h].double()
                s = s * fade + kk.t().contiguous() @ vv
                a = a * fade + kk.abs().t().contiguous() @ vv.abs()
                qq = q[b, lo:hi, qs].double()
                out[b, lo:hi, qs] = scale * (qq @ s)
                out_size[b, lo:hi, qs] = abs(scale) * (qq.abs() @ a)
            S[b, h], size[b, h] = s, a
        rounds.append(-(-m // per_round))
    return out, S, out_size, size, rounds


def linear_tolerances(want, out_size, size, rounds, per_round, D):
    """Bounds on out and state.  A decay over t rounds is a product or an exponential: its relative error is 4 u and 2 u a round.
    A sum in fp32 loses one rounding a term of the chain: up to per_round terms and one a round in the state, D and up to 64 pairs in the
    output.  The parts of what is decayed hold 24 bits (one u); the state's and the pairs' parts in the output's products 16
    (2^-16 each, two of them); the output is rounded once."""
    R = max(rounds + [1])
    state = (per_round + 4 * R + 16) * U32 * size + 1e-37
    out = U16 * want.abs() + (2 * 2.0 ** -16 + (per_round + 4 * R + D + 96) * U32) * out_size + 1e-37
    return out, state
