"""Performance cases of what a stream of rounds keeps: an 8-bit cache with the attention that reads it, and the state of linear attention.

One token is one site of one round of a stream (or of a volume).  A pass is one
call of one operator (for int8 caches the write and the read of what it wrote)
with everything resident on the device.  ``run`` is either the operator's plain
form (elementary torch operations in 32 bits, rounded once at the end) or the
calls of the library's kernels; ``exact`` is its definition in 64 bits.

  write      a token's keys and values go to place (at + m) mod capacity of its stream's
             ring as 8-bit codes, x / scale rounded, scale = max |x| / 448 or / 127 (kept in
             32 bits) for each token and head, with the token's site; tokens of volume < 0
             are left out
  read       values code scale of the places from `at` on; 0 where there is no token
  attention8 softmax(cap tanh(scale q.k / cap) - slope dist) v, k and v in such a cache,
             over the places of the query's volume, optionally those up to its own round
             or in a prefix of rounds; grouped heads
  linear     out_n = scale q_n S_t(n), S_t = exp(-slope) S_(t-1) + sum over the tokens of round t
             of k v^T; rounds of `per_round` tokens; S goes in and comes out

Positions ("sites") are int32 rows (t, i, j, volume); volume < 0: no token.  The
grids are those of the library's workloads: (d+1) x (d+1) sites a round.
"""
import math

import torch

own = False

DEV = "cuda"
QMAX = {"e4m3": 448.0, "int8": 127.0}
CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def listed():
    return [
        # one round of one d = 5 stream into its ring and back: the latency of two calls
        dict(name="write_d5_int8", op="write", batch=1, tokens=36, capacity=720, kv_heads=4, width=32, codes="int8", dtype="bf16", ragged=False),
        # the newest round of 64 streams of d = 13, out of the rows of the joint projection; some streams have none
        dict(name="write_d13_b64_e4m3", op="write", batch=64, tokens=196, capacity=2548, kv_heads=8, width=64, codes="e4m3", dtype="bf16", ragged=True),
        # four caches of up to 200 rounds of d = 13 read back, as a hand-over to a kernel of wide values
        dict(name="read_d13_e4m3", op="read", batch=4, tokens=39200, capacity=39200, kv_heads=2, width=64, codes="e4m3", dtype="bf16", ragged=True),
        # an odd range across the ring's end, in full precision
        dict(name="read_odd_int8", op="read", batch=3, tokens=1001, capacity=1501, kv_heads=3, width=48, codes="int8", dtype="fp32", ragged=False),
        # one round of a d = 5 stream against the twenty that it keeps
        dict(name="attention8_d5_round", op="attention8", batch=1, d=5, T=20, new=36, heads=4, kv_heads=4, width=32, codes="int8", cap=20.0, bias=True, causal=True, prefix=0),
        # one new token for each of four streams of d = 13 against up to 200 rounds
        dict(name="attention8_d13_token", op="attention8", batch=4, d=13, T=200, new=1, heads=8, kv_heads=2, width=64, codes="e4m3", cap=30.0, bias=True, causal=True, prefix=0),
        # a whole new round for each of them
        dict(name="attention8_d13_round", op="attention8", batch=4, d=13, T=200, new=196, heads=8, kv_heads=2, width=64, codes="e4m3", cap=30.0, bias=True, causal=True, prefix=0),
        # one token of sixteen streams of d = 15 with wide heads, every round in sight
        dict(name="attention8_d15_wide", op="attention8", batch=16, d=15, T=256, new=1, heads=8, kv_heads=2, width=128, codes="int8", cap=0.0, bias=False, causal=False, prefix=0),
        # one new round of a d = 5 stream: the state goes on by one
        dict(name="linear_d5_round", op="linear", batch=1, rounds=1, per_round=36, heads=4, kv_heads=4, width=32, ragged=False, state=True),
        # single tokens of 256 streams: the recurrent form
        dict(name="linear_token_b256", op="linear", batch=256, rounds=1, per_round=1, heads=8, kv_heads=8, width=128, ragged=False, state=True),
        # rows of single-token rounds of unequal odd lengths: the generic form
        dict(name="linear_rows_odd", op="linear", batch=8, rounds=4097, per_round=1, heads=6, kv_heads=6, width=64, ragged=True, state=True),
        # one stream of 1000 rounds of d = 13 taken in at once, grouped heads
        dict(name="linear_d13_stream", op="linear", batch=1, rounds=1000, per_round=196, heads=8, kv_heads=2, width=128, ragged=False, state=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["write", "read", "attention8", "attention8", "linear", "linear"])
    kv_heads = rng.choice([1, 2, 4, 8])
    width = rng.choice([32, 48, 64, 64, 96, 128])
    codes = rng.choice(["e4m3", "int8"])
    if op in ("write", "read"):
        batch = _log(rng, 1, 64)
        most = min(39200, 4 * 39200 * 2 * 64 // (batch * kv_heads * width))
        tokens = _log(rng, 1, max(2, most))
        return dict(op=op, batch=batch, tokens=tokens, capacity=tokens + rng.choice([0, 1, 196, tokens // 2]), kv_heads=kv_heads, width=width,
                    codes=codes, dtype=rng.choice(["bf16", "bf16", "fp32"]), ragged=rng.random() < 0.5)
    if op == "attention8":
        kv_heads = rng.choice([1, 2, 4])
        heads, d, batch = kv_heads * rng.choice([1, 2, 4]), rng.randrange(3, 24, 2), _log(rng, 1, 16)
        grid = (d + 1) ** 2
        new = rng.choice([1, 1, 7, grid])
        # at most the pairs of the listed round against its cache, and its bytes
        keys = min(4 * 8 * 196 * 39200 // (batch * heads * new), 16 * 65536 * 2 * 128 // (batch * kv_heads * width), 80000)
        causal = rng.random() < 0.6
        return dict(op=op, batch=batch, d=d, T=_log(rng, 1, max(2, keys // grid)), new=new, heads=heads, kv_heads=kv_heads, width=width, codes=codes,
                    cap=rng.choice([0.0, 15.0, 30.0, 50.0]), bias=rng.random() < 0.7, causal=causal, prefix=rng.choice([0, 0, 1, 3]) if causal else 0)
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    per_round = rng.choice([1, 1, 4, 9, 16, 36, 64, 100, 196, 324])
    batch = _log(rng, 1, 256)
    # at most the values of the listed stream, and its chunks of rounds in the plain form
    most = min(196000 * 10 * 128 // (batch * (heads + kv_heads) * width) // per_round, 1000 * max(1, 128 // per_round), 8192)
    return dict(op=op, batch=batch, rounds=_log(rng, 1, max(1, most)), per_round=per_round, heads=heads, kv_heads=kv_heads, width=width,
                ragged=rng.random() < 0.4, state=rng.random() < 0.6)


# ---- what a user has in hand ----


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (seed + 1))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _dtype(name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def _grid(d, T):
    """The sites of T rounds in (t, i, j) order, of volume 0."""
    t, i, j = torch.meshgrid(torch.arange(T, device=DEV), torch.arange(d + 1, device=DEV), torch.arange(d + 1, device=DEV), indexing="ij")
    return torch.stack([t, i, j, torch.zeros_like(t)], -1).reshape(-1, 4).to(torch.int32)


def _lengths(case):
    """Rounds in the cache (tokens of the call) of each stream: the last one is full, the others shorter."""
    T, B = case["T"], case["batch"]
    return [max(1, T * (b + 1 + B) // (2 * B)) for b in range(B)]


def _ragged(case, n):
    """Tokens of each stream: all, or for ragged streams none for some and up to all for the others."""
    B = case["batch"]
    if not case["ragged"]:
        return [n] * B
    return [n if b == B - 1 else 0 if b % 8 == 3 else n - (n * (b % 5)) // 11 for b in range(B)]


def _quantised(x, codes):
    """Codes and scales of the rows of x, for caches that are there before the call."""
    scale = x.abs().amax(-1) / QMAX[codes]
    y = x / torch.where(scale > 0, scale, 1.0)[..., None]
    return (y.round() if codes == "int8" else y).to(CODE[codes]), scale


def _cache(g, case, capacity):
    """Codes [batch][keys, values][head][place][width] and their scales [batch][2][head][place]; no sites yet."""
    B, Hk, D = case["batch"], case["kv_heads"], case["width"]
    codes = torch.empty(B, 2, Hk, capacity, D, device=DEV, dtype=CODE[case["codes"]])
    scales = torch.empty(B, 2, Hk, capacity, device=DEV)
    for b in range(0, B, 4):
        shape = codes[b:b + 4].shape
        codes[b:b + 4], scales[b:b + 4] = _quantised(_normal(g, *shape) * torch.exp(0.5 * _normal(g, *shape[:4], 1)), case["codes"])
    return codes, scales


def _by_token(cache):
    """Codes and scales of keys and of values, [batch][place][head][width] and [batch][place][head], and the sites."""
    codes, scales, sites = cache
    return [x[:, n].transpose(1, 2) for n in range(2) for x in (codes, scales)] + [sites]


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    B, Hk, D = case["batch"], case["kv_heads"], case["width"]
    if case["op"] in ("write", "read"):
        n, capacity = case["tokens"], case["capacity"]
        rest = _cache(g, case, capacity)
        at = torch.randint(0, capacity, (B,), generator=g, device=DEV)
        at[0] = capacity - (n + 1) // 2  # across the ring's end
        s["at"] = at
        place = torch.arange(capacity, device=DEV)
        length = torch.tensor(_ragged(case, n), device=DEV)
        m = torch.arange(n, device=DEV)
        first = torch.randint(0, 1000, (1,), generator=g, device=DEV)
        if case["op"] == "write":
            # the ring holds older tokens; the new ones come in the rows of the joint projection, with queries in front
            there = torch.ones(B, capacity, dtype=torch.bool, device=DEV)
            kv = _normal(g, B, n, Hk + 2 * Hk, D) * torch.exp(0.5 * _normal(g, B, n, 3 * Hk, 1))
            kv = kv.to(_dtype(case["dtype"]))
            s["k"], s["v"] = kv[:, :, Hk:2 * Hk], kv[:, :, 2 * Hk:]
            new = torch.where(m[None] < length[:, None], torch.arange(B, device=DEV)[:, None], -1)
            s["sites"] = torch.stack([(first + 1000).expand(B, n), (m // 64).expand(B, n), (m % 64).expand(B, n), new], -1).to(torch.int32)
        else:
            # tokens from `at` on, as many as the stream has
            there = (place[None] - at[:, None]) % capacity < length[:, None]
        volume = torch.where(there, torch.arange(B, device=DEV)[:, None], -1)
        sites = torch.stack([(first + place // 64).expand(B, capacity), (place % 8).expand(B, capacity), (place // 8 % 8).expand(B, capacity),
                             volume], -1).to(torch.int32)
        s["cache"] = (*rest, sites)
        if case["op"] == "read" or case["codes"] == "int8":
            s["k_out"], s["v_out"] = (torch.empty(B, n, Hk, D, device=DEV, dtype=_dtype(case["dtype"])) for _ in range(2))
    elif case["op"] == "attention8":
        grid, H, n = (case["d"] + 1) ** 2, case["heads"], case["new"]
        capacity = case["T"] * grid
        rest = _cache(g, case, capacity)
        last = torch.tensor(_lengths(case), device=DEV)
        sites = _grid(case["d"], case["T"]).repeat(B, 1, 1)
        volume = torch.arange(B, device=DEV, dtype=torch.int32)[:, None]
        sites[..., 3] = torch.where(sites[..., 0] < last[:, None], volume, -1)
        # the newest tokens: the first `new` sites of each stream's last round
        at = (last - 1)[:, None] * grid + torch.arange(n, device=DEV)[None]
        s["q_sites"] = torch.gather(sites, 1, at[..., None].expand(-1, -1, 4))
        # rings: a full cache begins in its middle
        turn = capacity // 2 + 7
        sites = sites.roll(turn, 1)
        s["cache"] = (*rest, sites.contiguous())
        s["q"] = (1.5 * _normal(g, B, n, H, D)).to(torch.bfloat16)
        s["slopes"] = torch.exp2(-8.0 * (torch.arange(H, device=DEV) + 1.0) / H) if case["bias"] else None
        s["out"] = torch.empty(B, n, H, D, device=DEV, dtype=torch.bfloat16)
        s["scale"] = 1.0 / math.sqrt(D)
    else:
        H, n = case["heads"], case["rounds"] * case["per_round"]
        # queries, keys and values in the rows of one joint projection
        qkv = torch.empty(B, n, H + 2 * Hk, D, device=DEV, dtype=torch.bfloat16)
        for b in range(0, B, 64):
            qkv[b:b + 64] = _normal(g, *qkv[b:b + 64].shape)
        s["q"], s["k"], s["v"] = qkv[:, :, :H], qkv[:, :, H:H + Hk], qkv[:, :, H + Hk:]
        s["slopes"] = torch.exp2(-8.0 * (torch.arange(Hk, device=DEV) + 1.0) / Hk)
        s["out"] = torch.zeros(B, n, H, D, device=DEV, dtype=torch.bfloat16)
        # what earlier rounds left, as large as this many tokens make it
        s["state"] = 4.0 * _normal(g, B, Hk, D, D) if case["state"] else None
        s["state_out"] = torch.empty(B, Hk, D, D, device=DEV, dtype=torch.float32)
        s["length"] = _ragged(case, n)
        s["lengths"] = torch.tensor(s["length"], device=DEV, dtype=torch.int32) if case["ragged"] else None
        s["scale"] = 1.0 / math.sqrt(D)
    return s


# ---- one pass ----


def run(s):
    case = s["case"]
    return (RUN_OWN if own else RUN_PLAIN)[case["op"]](s, case)


def _own_write(s, case):
    import paper_2604_12841_amd as pdx
    pdx.cache_write(s["cache"], s["at"], s["k"], s["v"], s["sites"])
    codes, scales, sites = s["cache"]
    if case["codes"] == "int8":
        # the values that the codes stand for
        pdx.cache_read(s["cache"], s["at"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"], "scales": scales, "sites": sites}
    return {"codes": codes, "scales": scales, "sites": sites}


def _places(s, case):
    """The place of each token, [batch][tokens]."""
    return (s["at"][:, None] + torch.arange(case["tokens"], device=DEV)) % case["capacity"]


def _plain_write(s, case):
    kc, ks, vc, vs, sites = _by_token(s["cache"])
    place = _places(s, case)
    b = torch.arange(case["batch"], device=DEV)[:, None]
    there = s["sites"][..., 3] >= 0
    for x, codes, scales in ((s["k"].float(), kc, ks), (s["v"].float(), vc, vs)):
        scale = x.abs().amax(-1)
        scale = scale / torch.full_like(scale, QMAX[case["codes"]])
        # the quotient in 64 bits: many lie next to the middle between two codes
        y = x.double() / torch.where(scale > 0, scale, 1.0)[..., None].double()
        if case["codes"] == "e4m3":
            step = torch.ldexp(torch.ones_like(y), torch.clamp(torch.frexp(y).exponent - 1, min=-6) - 3)
            y = torch.round(y / step) * step
        else:
            y = torch.round(y)
        y = y.float().to(CODE[case["codes"]]).view(torch.uint8)
        bits = codes.view(torch.uint8)
        bits[b, place] = torch.where(there[..., None, None], y, bits[b, place])
        scales[b, place] = torch.where(there[..., None], scale, scales[b, place])
    sites[b, place] = torch.where(there[..., None], s["sites"], sites[b, place])
    if case["codes"] == "int8":
        r = _plain_read(s, case)
        return {"k": r["k"], "v": r["v"], "scales": s["cache"][1], "sites": sites}
    return {"codes": s["cache"][0], "scales": s["cache"][1], "sites": sites}


def _own_read(s, case):
    import paper_2604_12841_amd as pdx
    pdx.cache_read(s["cache"], s["at"], s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_read(s, case):
    kc, ks, vc, vs, sites = _by_token(s["cache"])
    place = _places(s, case)
    b = torch.arange(case["batch"], device=DEV)[:, None]
    there = sites[b, place][..., 3] >= 0
    out = []
    for codes, scales in ((kc, ks), (vc, vs)):
        y = codes.view(torch.uint8)[b, place].view(codes.dtype).float() * scales[b, place][..., None]
        out.append(torch.where(there[..., None, None], y, 0.0).to(s["k_out"].dtype))
    return {"k": out[0], "v": out[1]}


def _own_attention8(s, case):
    import paper_2604_12841_amd as pdx
    pdx.attention8(s["q"], s["cache"], s["out"], s["q_sites"], scale=s["scale"], cap=case["cap"], slopes=s["slopes"], causal=case["causal"],
                   prefix=case["prefix"])
    return s["out"]


def _plain_attention8(s, case):
    kc, ks, vc, vs, k_sites = _by_token(s["cache"])
    group = case["heads"] // case["kv_heads"]
    q = s["q"].float().transpose(1, 2)
    k, v = ((c.float() * x[..., None]).transpose(1, 2).repeat_interleave(group, 1).contiguous() for c, x in ((kc, ks), (vc, vs)))
    score = torch.matmul(q.contiguous(), k.transpose(2, 3).contiguous()).mul_(s["scale"])
    if case["cap"] > 0:
        score = score.div_(case["cap"]).tanh_().mul_(case["cap"])
    a, b = s["q_sites"][:, :, None, :], k_sites[:, None, :, :]
    if case["bias"]:
        far = (a[..., 0] - b[..., 0]).abs() + (a[..., 1] - b[..., 1]).abs() + (a[..., 2] - b[..., 2]).abs()
        score = score.sub_(s["slopes"][:, None, None] * far[:, None].float())
    seen = (a[..., 3] == b[..., 3]) & (b[..., 3] >= 0)
    if case["causal"]:
        seen = seen & ((b[..., 0] <= a[..., 0]) | (b[..., 0] < case["prefix"]))
    score = score.masked_fill_(~seen[:, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return out.transpose(1, 2).contiguous().to(torch.bfloat16)


def _own_linear(s, case):
    import paper_2604_12841_amd as pdx
    pdx.linear_attention(s["q"], s["k"], s["v"], s["out"], slopes=s["slopes"], per_round=case["per_round"], lengths=s["lengths"], state=s["state"],
                         state_out=s["state_out"], scale=s["scale"])
    return {"out": s["out"], "state": s["state_out"]}


def _plain_linear(s, case):
    """Chunks of whole rounds: pairs inside a chunk, the state for what lies before it."""
    B, Hk, D, g, n = case["batch"], case["kv_heads"], case["width"], case["per_round"], case["rounds"] * case["per_round"]
    group = case["heads"] // Hk
    step = g * max(1, 128 // g)
    length = torch.tensor(s["length"], device=DEV) if s["lengths"] is None else s["lengths"].long()
    rounds = (length + g - 1) // g
    slope = s["slopes"].double()[:, None]  # (weights of far rounds: the exponent in 64 bits)
    S = s["state"].clone() if s["state"] is not None else torch.zeros(B, Hk, D, D, device=DEV)
    for lo in range(0, n, step):
        hi = min(n, lo + step)
        t = torch.arange(lo, hi, device=DEV) // g
        here = (torch.arange(lo, hi, device=DEV)[None] < length[:, None])[:, None, :, None]
        k, v = (torch.where(here, x[:, lo:hi].transpose(1, 2).float(), 0.0).contiguous() for x in (s["k"], s["v"]))
        q = s["q"][:, lo:hi].float().transpose(1, 2).reshape(B, Hk, group, hi - lo, D).contiguous()
        far = t[:, None] - t[None]
        weight = torch.where(far >= 0, torch.exp(-slope[..., None] * far.clamp(min=0)), 0.0).float()  # [Hk][..][..]
        pairs = torch.matmul(q, k.transpose(2, 3).contiguous()[:, :, None]) * weight[:, None]
        since = torch.exp(-slope * (t - lo // g + 1)).float()[:, None, :, None]
        out = torch.matmul(pairs, v[:, :, None]) + since * torch.matmul(q, S[:, :, None])
        out = (out * s["scale"]).reshape(B, Hk * group, hi - lo, D).transpose(1, 2).to(torch.bfloat16)
        s["out"][:, lo:hi] = torch.where(here.transpose(1, 2), out, s["out"][:, lo:hi])
        # rounds of this chunk that each entry has
        last = torch.clamp(rounds[:, None] - lo // g, min=0, max=(hi - lo) // g)
        left = torch.exp(-slope * torch.clamp(last[:, None] - 1 - (t - lo // g), min=0)).float()  # [B][Hk][..]
        S = S * torch.exp(-slope * last[:, None]).float()[..., None] + torch.matmul((k * left[..., None]).transpose(2, 3).contiguous(), v)
    s["state_out"].copy_(S)
    return {"out": s["out"], "state": s["state_out"]}


RUN_OWN = {"write": _own_write, "read": _own_read, "attention8": _own_attention8, "linear": _own_linear}
RUN_PLAIN = {"write": _plain_write, "read": _plain_read, "attention8": _plain_attention8, "linear": _plain_linear}


def work(case):
    B, Hk, D = case["batch"], case["kv_heads"], case["width"]
    if case["op"] in ("write", "read"):
        tokens, e = sum(_ragged(case, case["tokens"])), 2 if case["dtype"] == "bf16" else 4
        n, whole = 2 * tokens * Hk * D, 2 * B * case["tokens"] * Hk * D  # values of k and v; what a read writes, empty places too
        held = n + 8 * tokens * Hk + 16 * tokens  # codes, scales, sites
        if case["op"] == "read":
            return {"bytes": held + e * whole, "flops": n}
        back = e * whole if case["codes"] == "int8" else 0
        return {"bytes": e * n + held + 16 * B * case["tokens"] - 16 * tokens + 16 * tokens + back, "flops": 4 * n}
    if case["op"] == "attention8":
        grid, nq, H = (case["d"] + 1) ** 2, B * case["new"], case["heads"]
        # the newest tokens are in the last round of the cache: they see all of it
        keys = sum(_lengths(case)) * grid
        return {"bytes": 4 * nq * H * D + 16 * nq + keys * (Hk * (2 * D + 8) + 16), "flops": 4 * D * H * case["new"] * keys}
    tokens, H = sum(_ragged(case, case["rounds"] * case["per_round"])), case["heads"]
    states = 4 * B * Hk * D * D * (2 if case["state"] else 1)
    return {"bytes": 2 * tokens * D * (2 * H + 2 * Hk) + states, "flops": 2 * D * D * tokens * (H + Hk)}


# ---- the definitions in 64 bits ----


def exact(case, seed):
    s = prepare(case, seed)
    return EXACT[case["op"]](s, case)


def _e4m3(v):
    """v rounded to the nearest value with 3 mantissa bits and exponents from -6 (ties to even), at most 448."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.clamp(torch.round(v / step) * step, -448.0, 448.0)


def _exact_write(s, case):
    codes, scales, sites = (x.clone() for x in s["cache"])
    codes, scales = codes.double(), scales.double()
    n, whole = case["tokens"], case["codes"] == "int8"
    values = torch.zeros(2, case["batch"], n, case["kv_heads"], case["width"], device=DEV, dtype=torch.float64)
    for b in range(case["batch"]):
        there = (s["sites"][b, :, 3] >= 0).nonzero().flatten()
        place = (s["at"][b] + there) % case["capacity"]
        sites[b, place] = s["sites"][b, there]
        every = (s["at"][b] + torch.arange(n, device=DEV)) % case["capacity"]
        on = (sites[b, every, 3] >= 0)[:, None, None]
        for m, x in enumerate((s["k"], s["v"])):
            x = x[b, there].double().transpose(0, 1)
            scale = (torch.amax(torch.abs(x), -1) / QMAX[case["codes"]]).float().double()  # (codes go by the scale that is kept)
            y = x / scale[..., None]
            codes[b, m][:, place], scales[b, m][:, place] = torch.round(y) if whole else _e4m3(y), scale
            values[m, b] = torch.where(on, (codes[b, m] * scales[b, m][..., None]).transpose(0, 1)[every], 0.0)
    return {"k": values[0], "v": values[1], "scales": scales, "sites": sites} if whole else {"codes": codes, "scales": scales, "sites": sites}


def _exact_read(s, case):
    kc, ks, vc, vs, sites = _by_token(s["cache"])
    out = {}
    for n, codes, scales in (("k", kc, ks), ("v", vc, vs)):
        y = torch.zeros_like(s["k_out"], dtype=torch.float64)
        for b in range(case["batch"]):
            place = (s["at"][b] + torch.arange(case["tokens"], device=DEV)) % case["capacity"]
            on = (sites[b, place, 3] >= 0).nonzero().flatten()
            y[b, on] = codes[b].double()[place[on]] * scales[b, place[on]].double()[..., None]
        out[n] = y
    return out


def _exact_attention8(s, case):
    kc, ks, vc, vs, k_sites = _by_token(s["cache"])
    B, nq, H, D = s["q"].shape
    group = H // case["kv_heads"]
    out = torch.zeros(B, nq, H, D, device=DEV, dtype=torch.float64)
    for b in range(B):
        a, c = s["q_sites"][b], k_sites[b]
        seen = (a[:, None, 3] == c[None, :, 3]) & (c[None, :, 3] >= 0)
        if case["causal"]:
            seen &= (c[None, :, 0] <= a[:, None, 0]) | (c[None, :, 0] < case["prefix"])
        far = sum(torch.abs(a[:, None, axis] - c[None, :, axis]) for axis in range(3)).double()
        for h in range(H):
            k = kc[b, :, h // group].double() * ks[b, :, h // group].double()[:, None]
            v = vc[b, :, h // group].double() * vs[b, :, h // group].double()[:, None]
            z = torch.mm(s["q"][b, :, h].double(), k.t().contiguous()) * s["scale"]
            if case["cap"] > 0:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if s["slopes"] is not None:
                z = z - s["slopes"][h].double() * far
            z = torch.where(seen, z, -math.inf)
            top = z.amax(1, keepdim=True)
            p = torch.exp(z - torch.where(torch.isinf(top), 0.0, top))
            total = p.sum(1, keepdim=True)
            out[b, :, h] = torch.mm(p, v) / torch.where(total > 0, total, 1.0)
    return out


def _exact_linear(s, case):
    """Round by round."""
    B, Hk, D, g = case["batch"], case["kv_heads"], case["width"], case["per_round"]
    H = case["heads"]
    out = s["out"].double()
    S = s["state"].double() if s["state"] is not None else torch.zeros(B, Hk, D, D, device=DEV, dtype=torch.float64)
    fade = torch.exp(-s["slopes"].double())[None, :, None, None]
    length = torch.tensor(s["length"], device=DEV)
    for t in range(case["rounds"]):
        on = ((t * g + torch.arange(g, device=DEV))[None] < length[:, None])[..., None, None]
        k, v = (torch.where(on, x[:, t * g:(t + 1) * g].double(), 0.0).transpose(1, 2) for x in (s["k"], s["v"]))
        S = torch.where((t * g < length)[:, None, None, None], S * fade + torch.matmul(k.transpose(2, 3).contiguous(), v.contiguous()), S)
        q = s["q"][:, t * g:(t + 1) * g].double().transpose(1, 2).reshape(B, Hk, H // Hk * g, D)
        o = (s["scale"] * torch.matmul(q, S)).reshape(B, H, g, D).transpose(1, 2)
        out[:, t * g:(t + 1) * g] = torch.where(on, o, out[:, t * g:(t + 1) * g])
    return {"out": out, "state": S}


EXACT = {"write": _exact_write, "read": _exact_read, "attention8": _exact_attention8, "linear": _exact_linear}
