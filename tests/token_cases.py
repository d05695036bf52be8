"""Plain 64-bit forms of the token operators, and bounds on what their kernels may differ by."""
import math

import torch

U16, U32 = 2.0 ** -8, 2.0 ** -24  # largest relative error of one rounding to bf16 / fp32
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
UNIT = {torch.bfloat16: U16, torch.float32: U32}
EPS = 1e-6


def gen(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device=g.device, dtype=torch.float32)


# ---- norm ----

# A row's sum of squares is a chain of at most 32 products in a lane and 10 levels (lanes, waves) above it: relative error (32 + 10) u,
# halved by the root; mean, eps, root, reciprocal and the two products with s and gain add 6 u, s = x + r one.
NORM_REL = 28 * U32


def norm64(x, residual, gain):
    """(s, y) in 64 bits."""
    s = x.double() if residual is None else x.double() + residual.double()
    y = s / torch.sqrt((s * s).mean(1, keepdim=True) + EPS)
    return s, y if gain is None else y * gain.double()


def check_codes(codes, scales, y):
    """codes scales stands for y to half a step of the format, and the scale is the largest |y| over the format's largest value."""
    int8 = codes.dtype == torch.int8
    q = 127.0 if int8 else 448.0
    want = y.abs().amax(1) / q
    assert torch.all((scales.double() - want).abs() <= (NORM_REL + 2 * U32) * want)
    v = codes.double()
    assert torch.all(v.abs() <= q)
    t = y / torch.where(want > 0, want, 1.0)[:, None]
    # half a step: 1/2; E4M3: 2^-4 of the value, or 2^-10 below the normal range (2^-6)
    half = torch.full_like(t, 0.5) if int8 else torch.clamp(t.abs() * 2.0 ** -4, min=2.0 ** -10)
    assert torch.all((v - t).abs() <= half + 4 * NORM_REL * t.abs())


# ---- product ----


def matmul64(a, sa, w, sw, bias, act):
    """(result, sum of |products| with the scales) in 64 bits."""
    a, w = a.double(), w.double()
    scale = sa.double()[:, None] * sw.double()
    y = (a @ w.t().contiguous()) * scale
    size = (a.abs() @ w.abs().t().contiguous()) * scale.abs()
    if bias is not None:
        y = y + bias.double()
    if act == "gelu":
        y = y / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
    elif act == "relu":
        y = torch.clamp(y, min=0.0)
    return y, size


def matmul_tolerance(want, size, bias, int8, out_dtype, K):
    """The sum's error (int8: none but its conversion; E4M3 to bf16: 2^-16 of the sum of |products|, what the fp8 matrix
    instruction keeps; E4M3 to fp32: one fp32 rounding a product), scales, product and bias (4 roundings), the
    activation (slope at most 1.13, own error under 40 u) and the output's rounding."""
    part = U32 if int8 else K * U32 if out_dtype == torch.float32 else 2.0 ** -16 + K / 64 * U32
    b = 0.0 if bias is None else bias.double().abs()
    return 1.13 * (part * size + 4 * U32 * (size + b)) + (40 * U32 + UNIT[out_dtype]) * want.abs() + 1e-30


# ---- rotary positions ----


def rope64(x, sites, sections, base, interleaved, inverse):
    x, p = x.double(), sites.double()
    P = x.shape[-1] // 2
    out = x.clone()
    m = 0
    for axis, n in enumerate(sections):
        for k in range(n):
            u, v = (2 * m, 2 * m + 1) if interleaved else (m, m + P)
            angle = p[:, axis, None] * base ** (-k / n) * (-1 if inverse else 1)
            c, s = torch.cos(angle), torch.sin(angle)
            out[..., u] = x[..., u] * c - x[..., v] * s
            out[..., v] = x[..., v] * c + x[..., u] * s
            m += 1
    return out


def rope_tolerance(x, want, interleaved):
    """The angle is within 2 x 2^-24 turns; sine and cosine to fp32 within 4 u of it, for bf16 results within 2^-14 (64
    times finer than their rounding); two products, one sum."""
    h = x.double().abs()
    P = x.shape[-1] // 2
    pair = (h[..., 0::2] + h[..., 1::2]).repeat_interleave(2, -1) if interleaved else \
        (h[..., :P] + h[..., P:]).repeat(1, 1, 2)
    part = 4 * math.pi * U32 + 7 * U32 if x.dtype == torch.float32 else 2.0 ** -14
    return part * pair + UNIT[x.dtype] * want.abs()


# ---- attention ----


def attention64(q, k, v, q_sites, k_sites, scale, cap, slopes, causal, prefix):
    """(out, what a unit of error in the probabilities moves it by, the largest score error) in 64 bits."""
    B, nq, H, D = q.shape
    nk, Hk = k.shape[1], k.shape[2]
    q, k, v = (x.double().transpose(1, 2) for x in (q, k, v))
    k, v = (x.repeat_interleave(H // Hk, 1) for x in (k, v))
    z = (q @ k.transpose(2, 3).contiguous()) * scale
    size = (q.abs().nan_to_num(0, 0, 0) @ k.abs().nan_to_num(0, 0, 0).transpose(2, 3).contiguous()) * abs(scale)
    if cap > 0:
        z = cap * torch.tanh(z / cap)
    seen = torch.ones(B, 1, nq, nk, dtype=torch.bool, device=z.device)
    far = 0.0
    if q_sites is not None:
        a = q_sites.expand(B, nq, 4)[:, None, :, None, :].long()
        b = k_sites.expand(B, nk, 4)[:, None, None, :, :].long()
        if slopes is not None:
            far = (a[..., :3] - b[..., :3]).abs().sum(-1).double() * slopes.double()[None, :, None, None]
            z = z - far
        seen = (a[..., 3] == b[..., 3]) & (b[..., 3] >= 0)
        if causal:
            seen = seen & ((b[..., 0] <= a[..., 0]) | (b[..., 0] < prefix))
    z = torch.where(seen, z, -math.inf)
    if nk == 0:
        zero = torch.zeros(B, nq, H, D, dtype=torch.float64, device=z.device)
        return zero, zero, 0.0
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(torch.isneginf(top), 0.0, top))
    p = torch.where(seen, p, 0.0)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    # nothing of an invisible token, whatever it holds: its value counts as 0 where p is 0 for every row, and rows are
    # taken one by one where some see it
    clean = torch.nan_to_num(v, 0, 0, 0)
    out = p @ clean
    odd = ~torch.isfinite(v)
    if odd.any():
        for key in odd.any(3).any(1).any(0).nonzero().flatten().tolist():
            w = torch.where(odd[:, :, key], v[:, :, key], 0.0)[:, :, None, :]
            on = seen[..., key].expand(B, H, nq)[..., None]
            out = out + torch.where(on, p[..., key, None] * w, 0.0)
    moved = p @ clean.abs()
    # fp32 score: the product (D roundings at most), the cap (its parts are at most 2 cap), the distance
    score = torch.where(seen, (D * U32) * size, 0.0).nan_to_num(0, 0, 0).amax() + 8 * U32 * cap + \
        4 * U32 * (far.amax() if torch.is_tensor(far) else 0.0)
    return out.transpose(1, 2), moved.transpose(1, 2), float(score)


def attention_tolerance(want, moved, score):
    """Rounded probabilities (2^-8 each), scores off by `score` and their exponential (its argument, up to 2^7 log2 units that
    matter, rounded: 2^7 u; the instruction: 2 u), in the probabilities and in their sum; the result's rounding. The
    constant holds bf16's subnormal step."""
    return U16 * want.abs() + (U16 + 2 * (score + 130 * U32)) * moved * 1.01 + 1e-38
