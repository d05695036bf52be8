"""Performance cases of the token operators: what a block of attention over the sites of detector volumes runs.

One token is one site of one round of a volume.  A pass is one call of one
operator with everything resident on the device.  ``run`` is either the
operator's plain form (elementary torch operations in 32 bits, rounded once at
the end) or the call of the library's kernel; ``exact`` is its definition in 64
bits.

  norm       s = x + r;  y = s / sqrt(mean(s^2) + eps) * g, given as it is or in 8
             bits (E4M3 or int8 codes) with a scale for each token
  matmul     act(sa[m] sw[n] sum_k a[m][k] w[n][k] + b[n]) of 8-bit codes
  rope       rotary positions over the axes (round, row, column)
  attention  softmax(cap tanh(scale q.k / cap) - slope dist) v over the tokens of the
             same volume (dist: L1 distance of the sites), optionally those up
             to a token's own round or in a prefix of rounds; grouped heads

Positions ("sites") are int32 rows (t, i, j, volume); volume < 0 is padding.
The grids are those of the library's workloads: (d+1) x (d+1) sites, T rounds.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
BASE = 100.0
QMAX = {"e4m3": 448.0, "int8": 127.0}


def listed():
    return [
        # one small volume (d = 5, 5 rounds) through a 128-wide layer: the latency of a call
        dict(name="norm_d5_int8", op="norm", rows=180, width=128, dtype="bf16", residual=True, codes="int8", pad=0),
        # the residual stream of 64 volumes of d = 13, T = 13 on the way into an fp8 product
        dict(name="norm_d13_b64_e4m3", op="norm", rows=163072, width=512, dtype="bf16", residual=True, codes="e4m3", pad=0),
        # full precision, an odd width inside wider rows
        dict(name="norm_odd_fp32", op="norm", rows=9001, width=333, dtype="fp32", residual=False, codes="none", pad=19),
        # the output projection for one small volume: few rows
        dict(name="matmul_d5_int8", op="matmul", M=180, K=512, N=512, codes="int8", out="bf16", bias=True, act="none", pad=0),
        # the widening product of a block, with its activation, for 64 volumes of d = 13
        dict(name="matmul_d13_b64_e4m3", op="matmul", M=163072, K=512, N=2048, codes="e4m3", out="bf16", bias=True, act="gelu", pad=0),
        # a long sum to odd sizes in unaligned rows
        dict(name="matmul_odd_int8", op="matmul", M=7201, K=2047, N=771, codes="int8", out="fp32", bias=False, act="none", pad=3),
        # one round of a d = 5 stream, queries and keys of a narrow block
        dict(name="rope_d5_round", op="rope", tokens=36, heads=6, width=32, dtype="bf16", interleaved=False, inverse=False, d=5, extra=2),
        # queries and keys of 64 volumes of d = 13 inside the rows of the joint projection
        dict(name="rope_d13_b64", op="rope", tokens=163072, heads=10, width=64, dtype="bf16", interleaved=False, inverse=False, d=13, extra=2),
        # 64 small volumes in one batch, all pairs of a volume
        dict(name="attention_d5_b64", op="attention", kind="batch", d=5, T=5, batch=64, heads=4, kv_heads=4, width=32, cap=20.0, bias=True, causal=False, prefix=0),
        # 16 volumes of d = 13 with grouped heads
        dict(name="attention_d13_b16", op="attention", kind="batch", d=13, T=13, batch=16, heads=8, kv_heads=2, width=64, cap=30.0, bias=True, causal=False, prefix=0),
        # volumes of several distances packed in one row of tokens, rounds seen up to their own
        dict(name="attention_packed", op="attention", kind="packed", volumes="5x9,13x13,9x9,3x4,11x30,7x7,17x17,13x20", batch=1, heads=4, kv_heads=2, width=128, cap=0.0, bias=True, causal=True, prefix=2),
        # the newest tokens of four streams of d = 13 against their caches of up to 200 rounds
        dict(name="attention_step_cache", op="attention", kind="step", d=13, T=200, batch=4, new=1, heads=8, kv_heads=2, width=64, cap=30.0, bias=True, causal=True, prefix=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["norm", "matmul", "rope", "attention", "attention"])
    if op == "norm":
        width = rng.choice([64, 128, 256, 512, 512, 1024, 2048, _log(rng, 8, 2048)])
        rows = _log(rng, 1, min(163072, 163072 * 512 // width))
        codes = rng.choice(["none", "e4m3", "e4m3", "int8"])
        return dict(op=op, rows=rows, width=width, dtype=rng.choice(["bf16", "bf16", "fp32"]), residual=rng.random() < 0.6,
                    codes=codes, pad=rng.choice([0, 0, 0, 8, 5]))
    if op == "matmul":
        K, N = (rng.choice([128, 256, 512, 1024, 2048, _log(rng, 16, 2048)]) for _ in range(2))
        M = _log(rng, 1, min(163072, 163072 * 512 * 2048 // (K * N)))
        return dict(op=op, M=M, K=K, N=N, codes=rng.choice(["e4m3", "int8"]), out=rng.choice(["bf16", "bf16", "fp32"]),
                    bias=rng.random() < 0.5, act=rng.choice(["none", "none", "gelu", "relu"]), pad=rng.choice([0, 0, 0, 16, 3]))
    if op == "rope":
        heads, width = rng.randrange(1, 17), rng.choice([32, 48, 64, 64, 96, 128])
        return dict(op=op, tokens=_log(rng, 1, min(163072, 163072 * 640 // (heads * width))), heads=heads, width=width,
                    dtype=rng.choice(["bf16", "bf16", "fp32"]), interleaved=rng.random() < 0.4, inverse=rng.random() < 0.3,
                    d=rng.randrange(3, 32, 2), extra=rng.choice([0, 2, 5]))
    kv_heads = rng.choice([1, 2, 4])
    heads = kv_heads * rng.choice([1, 2, 4])
    c = dict(op=op, kind=rng.choice(["batch", "packed", "step"]), batch=1, heads=heads, kv_heads=kv_heads,
             width=rng.choice([32, 48, 64, 64, 96, 128]), cap=rng.choice([0.0, 15.0, 30.0, 50.0]), bias=rng.random() < 0.7,
             causal=rng.random() < 0.5, prefix=0)
    most = 16 * 8 * 2548 ** 2 // 2  # pairs of tokens and heads in the largest listed case, and some room
    if c["kind"] == "batch":
        c["d"] = rng.randrange(3, 18, 2)
        c["T"] = rng.randrange(1, 18)
        n = c["T"] * (c["d"] + 1) ** 2
        c["batch"] = _log(rng, 1, max(1, min(128, most // (heads * n * n))))
    elif c["kind"] == "packed":
        todo, at = _log(rng, 200, min(9000, math.isqrt(most // heads))), []
        while todo > 0:
            d, T = rng.randrange(3, 18, 2), rng.randrange(1, 24)
            at.append("%dx%d" % (d, T))
            todo -= T * (d + 1) ** 2
        c["volumes"] = ",".join(at[:24])
    else:
        c.update(d=rng.randrange(3, 24, 2), causal=True)
        c["T"] = _log(rng, 2, max(3, min(1000, 80000 // (c["d"] + 1) ** 2)))
        c["new"] = rng.choice([1, 1, 7, (c["d"] + 1) ** 2])
        c["batch"] = _log(rng, 1, 8)
    if c["causal"]:
        c["prefix"] = rng.choice([0, 0, 1, 3])
    return c


# ---- what a user has in hand ----


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (seed + 1))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _dtype(name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def _volume_sites(d, T, volume):
    """The sites of one volume in (t, i, j) order."""
    t, i, j = torch.meshgrid(torch.arange(T, device=DEV), torch.arange(d + 1, device=DEV), torch.arange(d + 1, device=DEV),
                             indexing="ij")
    return torch.stack([t, i, j, torch.full_like(t, volume)], -1).reshape(-1, 4).to(torch.int32)


def _volumes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["volumes"].split(",")]


def _lengths(case):
    """Rounds in the cache of each stream: the last one is full, the others shorter."""
    T, B = case["T"], case["batch"]
    return [max(1, T * (b + 1 + B) // (2 * B)) for b in range(B)]


def _shapes(case):
    """(batch, queries, keys) of an attention case."""
    if case["kind"] == "batch":
        n = case["T"] * (case["d"] + 1) ** 2
        return case["batch"], n, n
    if case["kind"] == "packed":
        n = sum(T * (d + 1) ** 2 for d, T in _volumes(case))
        return 1, n, n
    return case["batch"], case["new"], case["T"] * (case["d"] + 1) ** 2


def _pairs(case):
    """Visible pairs of tokens."""
    def volume(d, T, rounds_seen):
        g = (d + 1) ** 2
        return sum(g * g * rounds_seen(t) for t in range(T))

    def seen(T):
        return (lambda t: min(T, max(t + 1, case["prefix"]))) if case["causal"] else (lambda t: T)
    if case["kind"] == "batch":
        return case["batch"] * volume(case["d"], case["T"], seen(case["T"]))
    if case["kind"] == "packed":
        return sum(volume(d, T, seen(T)) for d, T in _volumes(case))
    # the newest tokens are in the last round of the cache: they see all of it
    return sum(case["new"] * n * (case["d"] + 1) ** 2 for n in _lengths(case))


def _sections(width):
    """Pairs for the rounds, the rows and the columns: a half and two quarters."""
    pairs = width // 2
    a = pairs // 4
    return pairs - 2 * a, a, a


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] == "norm":
        R, C, dt = case["rows"], case["width"], _dtype(case["dtype"])
        # activations of unequal size from token to token, a few large channels, as behind a GELU or a projection
        spread = torch.exp(0.7 * _normal(g, R, 1))
        channel = torch.exp(0.5 * _normal(g, C + case["pad"]))
        s["x"] = (_normal(g, R, C + case["pad"]) * spread * channel).to(dt)[:, :C]
        s["r"] = _normal(g, R, C).to(dt) if case["residual"] else None
        s["g"] = 1.0 + 0.2 * _normal(g, C)
        if case["residual"]:
            s["sum"] = torch.empty(R, C, device=DEV, dtype=dt)
        if case["codes"] == "none":
            s["out"] = torch.empty(R, C, device=DEV, dtype=dt)
        else:
            s["codes"] = torch.empty(R, C, device=DEV, dtype=torch.int8 if case["codes"] == "int8" else torch.float8_e4m3fn)
            s["scales"] = torch.empty(R, device=DEV, dtype=torch.float32)
        if case["codes"] == "int8":
            s["values"] = torch.empty(R, C, device=DEV, dtype=torch.bfloat16)
    elif case["op"] == "matmul":
        M, K, N = case["M"], case["K"], case["N"]

        def codes(rows):
            x = _normal(g, rows, K + case["pad"])
            q = QMAX[case["codes"]]
            x = x * (q / x.abs().amax(1, keepdim=True))  # each row uses the whole range
            return (x.round().to(torch.int8) if case["codes"] == "int8" else x.to(torch.float8_e4m3fn))[:, :K]
        s["a"], s["w"] = codes(M), codes(N)
        q = QMAX[case["codes"]]
        s["sa"] = torch.exp(0.5 * _normal(g, M)) * (4.0 / q)
        s["sw"] = torch.exp(0.3 * _normal(g, N)) * (4.0 / (q * math.sqrt(K)))
        s["bias"] = 0.35 * _normal(g, N) if case["bias"] else None
        s["out"] = torch.empty(M, N, device=DEV, dtype=_dtype(case["out"]))
    elif case["op"] == "rope":
        n, H, D = case["tokens"], case["heads"], case["width"]
        dt = _dtype(case["dtype"])
        s["x"] = _normal(g, n, H + case["extra"], D).to(dt)[:, :H]
        grid = (case["d"] + 1) ** 2
        at = torch.arange(n, device=DEV)
        first = torch.randint(0, 32, (1,), generator=g, device=DEV)  # the round at which the tokens begin
        T = 2 * case["d"]
        t = at // grid
        s["sites"] = torch.stack([first + t % T, at % grid // (case["d"] + 1), at % (case["d"] + 1), t // T], -1).to(torch.int32)
        s["out"] = torch.empty(n, H, D, device=DEV, dtype=dt)
    else:
        B, nq, nk = _shapes(case)
        H, Hk, D = case["heads"], case["kv_heads"], case["width"]
        if case["kind"] == "step":
            # the cache keeps keys and values of a token side by side; a stream's rest of it holds no tokens yet
            kv = _normal(g, B, nk, 2, Hk, D).to(torch.bfloat16)
            s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
            s["q"] = (1.5 * _normal(g, B, nq, H, D)).to(torch.bfloat16)
            sites = _volume_sites(case["d"], case["T"], 0).repeat(B, 1, 1)
            grid = (case["d"] + 1) ** 2
            last = torch.tensor(_lengths(case), device=DEV, dtype=torch.int32)
            volume = torch.arange(B, device=DEV, dtype=torch.int32)[:, None]
            sites[..., 3] = torch.where(sites[..., 0] < last[:, None], volume, -1)
            # the newest tokens: the first `new` sites of each stream's last round
            at = (last.long() - 1)[:, None] * grid + torch.arange(nq, device=DEV)[None]
            s["k_sites"] = sites
            s["q_sites"] = torch.gather(sites, 1, at[..., None].expand(-1, -1, 4))
            if nq > grid:
                raise ValueError("a step holds at most one round")
        else:
            # queries, keys and values in the rows of one joint projection
            qkv = _normal(g, B, nq, H + 2 * Hk, D)
            qkv[:, :, :H] *= 1.5
            qkv = qkv.to(torch.bfloat16)
            s["q"], s["k"], s["v"] = qkv[:, :, :H], qkv[:, :, H:H + Hk], qkv[:, :, H + Hk:]
            if case["kind"] == "batch":
                s["q_sites"] = _volume_sites(case["d"], case["T"], 0)
            else:
                s["q_sites"] = torch.cat([_volume_sites(d, T, n) for n, (d, T) in enumerate(_volumes(case))])
            s["k_sites"] = s["q_sites"]
        # one slope a head, a geometric run of them
        s["slopes"] = torch.exp2(-8.0 * (torch.arange(H, device=DEV) + 1.0) / H) if case["bias"] else None
        s["out"] = torch.empty(B, nq, H, D, device=DEV, dtype=torch.bfloat16)
        s["scale"] = 1.0 / math.sqrt(D)
    return s


# ---- one pass ----


def run(s):
    case = s["case"]
    return (RUN_OWN if own else RUN_PLAIN)[case["op"]](s, case)


def _own_norm(s, case):
    import paper_2604_12841_amd as pdx
    pdx.rms_norm(s["x"], s["g"], eps=EPS, residual=s["r"], sum_out=s.get("sum"), out=s.get("out"), codes=s.get("codes"),
                 scales=s.get("scales"))
    if case["codes"] == "int8":
        # the values that the codes stand for
        torch.mul(s["codes"], s["scales"][:, None], out=s["values"])
        return {"sum": s.get("sum"), "values": s["values"], "scales": s["scales"]}
    return {"sum": s.get("sum"), "out": s.get("out"), "codes": s.get("codes"), "scales": s.get("scales")}


def _plain_norm(s, case):
    x = s["x"].float()
    if case["residual"]:
        x = x + s["r"].float()
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * s["g"]
    total = x.to(s["x"].dtype) if case["residual"] else None
    if case["codes"] == "none":
        return {"sum": total, "out": y.to(s["x"].dtype), "codes": None, "scales": None}
    scales = y.abs().amax(1) / QMAX[case["codes"]]
    code = torch.where(scales[:, None] > 0, y / scales[:, None], 0.0)
    if case["codes"] == "int8":
        return {"sum": total, "values": (torch.round(code) * scales[:, None]).to(torch.bfloat16), "scales": scales}
    return {"sum": total, "out": None, "codes": code.to(torch.float8_e4m3fn), "scales": scales}


def _own_matmul(s, case):
    import paper_2604_12841_amd as pdx
    pdx.matmul8(s["a"], s["sa"], s["w"], s["sw"], s["out"], bias=s["bias"], act=case["act"])
    return s["out"]


def _plain_matmul(s, case):
    y = s["a"].float() @ s["w"].float().t()
    y = y * s["sa"][:, None] * s["sw"]
    if case["bias"]:
        y = y + s["bias"]
    if case["act"] == "gelu":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    elif case["act"] == "relu":
        y = torch.clamp(y, min=0.0)
    return y.to(s["out"].dtype)


def _own_rope(s, case):
    import paper_2604_12841_amd as pdx
    pdx.rope(s["x"], s["sites"], s["out"], _sections(case["width"]), base=BASE, interleaved=case["interleaved"],
             inverse=case["inverse"])
    return s["out"]


def _angles(s, case, dtype):
    """[token][pair]: the position on the pair's axis times its frequency."""
    at = s["sites"].to(dtype)
    return torch.cat([at[:, axis, None] * torch.pow(BASE, -torch.arange(n, device=DEV, dtype=dtype) / n)
                      for axis, n in enumerate(_sections(case["width"]))], 1)


def _turn(x, c, sn, interleaved):
    if interleaved:
        u, v = x[..., 0::2], x[..., 1::2]
        return torch.stack([u * c - v * sn, v * c + u * sn], -1).flatten(-2)
    u, v = x.chunk(2, -1)
    return torch.cat([u * c - v * sn, v * c + u * sn], -1)


def _plain_rope(s, case):
    a = _angles(s, case, torch.float32)
    a = -a if case["inverse"] else a
    return _turn(s["x"].float(), torch.cos(a)[:, None], torch.sin(a)[:, None], case["interleaved"]).to(s["x"].dtype)


def _own_attention(s, case):
    import paper_2604_12841_amd as pdx
    pdx.attention(s["q"], s["k"], s["v"], s["out"], q_sites=s["q_sites"], k_sites=s["k_sites"], scale=s["scale"],
                  cap=case["cap"], slopes=s["slopes"], causal=case["causal"], prefix=case["prefix"])
    return s["out"]


def _plain_attention(s, case):
    q, k, v = (s[n].float().transpose(1, 2) for n in "qkv")
    group = case["heads"] // case["kv_heads"]
    k, v = (x.repeat_interleave(group, 1).contiguous() for x in (k, v))
    score = torch.matmul(q.contiguous(), k.transpose(2, 3).contiguous()).mul_(s["scale"])
    if case["cap"] > 0:
        score = score.div_(case["cap"]).tanh_().mul_(case["cap"])
    a, b = s["q_sites"][..., :, None, :], s["k_sites"][..., None, :, :]
    if case["bias"]:
        far = (a[..., 0] - b[..., 0]).abs() + (a[..., 1] - b[..., 1]).abs() + (a[..., 2] - b[..., 2]).abs()
        score = score.sub_(s["slopes"][:, None, None] * (far if far.dim() == 2 else far[:, None]).float())
    seen = (a[..., 3] == b[..., 3]) & (b[..., 3] >= 0)
    if case["causal"]:
        seen = seen & ((b[..., 0] <= a[..., 0]) | (b[..., 0] < case["prefix"]))
    score = score.masked_fill_(~(seen if seen.dim() == 2 else seen[:, None]), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return out.transpose(1, 2).contiguous().to(torch.bfloat16)


RUN_OWN = {"norm": _own_norm, "matmul": _own_matmul, "rope": _own_rope, "attention": _own_attention}
RUN_PLAIN = {"norm": _plain_norm, "matmul": _plain_matmul, "rope": _plain_rope, "attention": _plain_attention}


def work(case):
    if case["op"] == "norm":
        n, e = case["rows"] * case["width"], 2 if case["dtype"] == "bf16" else 4
        each = e * (3 if case["residual"] else 1) + (e if case["codes"] == "none" else 1)
        return {"bytes": n * each + 4 * case["width"] + (0 if case["codes"] == "none" else 4 * case["rows"]), "flops": 8 * n}
    if case["op"] == "matmul":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": (M + N) * K + M * N * (2 if case["out"] == "bf16" else 4) + 4 * (M + N) + (4 * N if case["bias"] else 0),
                "flops": 2 * M * K * N}
    if case["op"] == "rope":
        n = case["tokens"] * case["heads"] * case["width"]
        return {"bytes": 2 * n * (2 if case["dtype"] == "bf16" else 4) + 16 * case["tokens"], "flops": 3 * n}
    B, nq, nk = _shapes(case)
    keys = sum(_lengths(case)) * (case["d"] + 1) ** 2 if case["kind"] == "step" else B * nk  # tokens that are there
    sites = 16 * (B * nq + B * nk if case["kind"] == "step" else nq)
    return {"bytes": 2 * case["width"] * (2 * B * nq * case["heads"] + 2 * keys * case["kv_heads"]) + sites,
            "flops": 4 * case["width"] * case["heads"] * _pairs(case)}


# ---- the definitions in 64 bits ----


def exact(case, seed):
    s = prepare(case, seed)
    return EXACT[case["op"]](s, case)


def _e4m3(v):
    """v rounded to the nearest value with 3 mantissa bits and exponents from -6 (ties to even), at most 448."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.clamp(torch.round(v / step) * step, -448.0, 448.0)


def _exact_norm(s, case):
    x = s["x"].double()
    if s["r"] is not None:
        x = x + s["r"].double()
    y = s["g"].double() * x / torch.sqrt(torch.sum(x ** 2, 1, keepdim=True) / case["width"] + EPS)
    total = x if case["residual"] else None
    if case["codes"] == "none":
        return {"sum": total, "out": y, "codes": None, "scales": None}
    scales = torch.amax(torch.abs(y), 1) / QMAX[case["codes"]]
    code = y / scales[:, None]
    if case["codes"] == "int8":
        return {"sum": total, "values": torch.round(code) * scales[:, None], "scales": scales}
    return {"sum": total, "out": None, "codes": _e4m3(code), "scales": scales}


def _exact_matmul(s, case):
    def rows(lo, hi):
        y = torch.mm(s["a"][lo:hi].to(torch.float64), s["w"].to(torch.float64).t().contiguous())
        y = torch.outer(s["sa"][lo:hi].double(), s["sw"].double()) * y
        if s["bias"] is not None:
            y += s["bias"].double()
        if case["act"] == "gelu":
            u = math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)
            y = y / (1.0 + torch.exp(-2.0 * u))
        elif case["act"] == "relu":
            y = torch.where(y > 0, y, 0.0)
        return y
    step = 32768
    return torch.cat([rows(m, min(m + step, case["M"])) for m in range(0, case["M"], step)])


def _exact_rope(s, case):
    x, at = s["x"].double(), s["sites"].double()
    pairs = case["width"] // 2
    out = torch.empty_like(x, memory_format=torch.contiguous_format)
    m = 0
    for axis, n in enumerate(_sections(case["width"])):
        for k in range(n):
            u, v = (2 * m, 2 * m + 1) if case["interleaved"] else (m, m + pairs)
            turn = (-1.0 if case["inverse"] else 1.0) * at[:, axis] * BASE ** (-k / n)
            c, sn = torch.cos(turn)[:, None], torch.sin(turn)[:, None]
            out[..., u] = x[..., u] * c - x[..., v] * sn
            out[..., v] = x[..., u] * sn + x[..., v] * c
            m += 1
    return out


def _exact_attention(s, case):
    B, nq, nk = _shapes(case)
    H, D = case["heads"], case["width"]
    group = H // case["kv_heads"]
    out = torch.zeros(B, nq, H, D, device=DEV, dtype=torch.float64)
    step = max(1, 2 ** 27 // nk)
    for b in range(B):
        qs = s["q_sites"] if s["q_sites"].dim() == 2 else s["q_sites"][b]
        ks = s["k_sites"] if s["k_sites"].dim() == 2 else s["k_sites"][b]
        for lo in range(0, nq, step):
            hi = min(nq, lo + step)
            seen = (qs[lo:hi, None, 3] == ks[None, :, 3]) & (ks[None, :, 3] >= 0)
            if case["causal"]:
                t, u = qs[lo:hi, None, 0], ks[None, :, 0]
                seen &= (u <= t) | (u < case["prefix"])
            far = sum(torch.abs(qs[lo:hi, None, axis] - ks[None, :, axis]) for axis in range(3)).double()
            for h in range(H):
                z = torch.mm(s["q"][b, lo:hi, h].double(), s["k"][b, :, h // group].double().t().contiguous()) * s["scale"]
                if case["cap"] > 0:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                if s["slopes"] is not None:
                    z = z - s["slopes"][h].double() * far
                z = torch.where(seen, z, -math.inf)
                top = z.amax(1, keepdim=True)
                p = torch.exp(z - torch.where(torch.isinf(top), 0.0, top))
                total = p.sum(1, keepdim=True)
                out[b, lo:hi, h] = torch.mm(p, s["v"][b, :, h // group].double()) / torch.where(total > 0, total, 1.0)
    return out


EXACT = {"norm": _exact_norm, "matmul": _exact_matmul, "rope": _exact_rope, "attention": _exact_attention}
