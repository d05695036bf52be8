"""GPU: the product of 8-bit codes against its definition in 64 bits."""
import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def codes(g, rows, K, kind, pad=0, shift=0):
    n = rows * (K + pad) + shift
    if kind == "int8":
        t = torch.randint(-127, 128, (n,), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    else:
        t = (tc.normal(g, n) * 60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
    return t[shift:].view(rows, K + pad)[:, :K]


def check(M, N, K, kind, out="bf16", bias=False, act="none", pad=0, shift=0, out_pad=0, seed=0):
    g = tc.gen(seed + M * 7 + N * 3 + K)
    a, w = codes(g, M, K, kind, pad, shift), codes(g, N, K, kind, pad, shift)
    q = (127.0 if kind == "int8" else 60.0)
    sa = torch.exp(0.3 * tc.normal(g, M)) / q
    sw = torch.exp(0.3 * tc.normal(g, N)) / (q * max(K, 1) ** 0.5)
    b = tc.normal(g, N) if bias else None
    whole = torch.full((M, N + out_pad), 5.0, dtype=tc.DTYPES[out], device="cuda")
    o = whole[:, :N]
    pdx.matmul8(a, sa, w, sw, o, bias=b, act=act)
    torch.cuda.synchronize()
    want, size = tc.matmul64(a, sa, w, sw, b, act)
    assert torch.all((o.double() - want).abs() <= tc.matmul_tolerance(want, size, b, kind == "int8", o.dtype, K))
    assert torch.all(whole[:, N:] == 5.0)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 512, 512), (3, 70, 16), (5, 8, 48), (16, 64, 64), (17, 16, 4096), (36, 128, 2048), (64, 64, 128),
                                   (65, 65, 65), (100, 771, 333), (128, 256, 512), (180, 512, 512), (255, 129, 80), (257, 511, 1040),
                                   (1000, 320, 576), (2548, 768, 256), (3, 2048, 8192), (4100, 520, 128)])
def test_sizes(M, N, K, kind, out):
    check(M, N, K, kind, out, bias=True)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("act", ["none", "gelu", "relu"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("M,N,K", [(40, 96, 160), (600, 512, 512)])
def test_epilogues(M, N, K, kind, act, bias):
    check(M, N, K, kind, "bf16", bias, act)
    check(M, N, K, kind, "fp32", bias, act)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("pad,shift,out_pad", [(16, 0, 0), (0, 1, 0), (3, 0, 5), (1, 7, 1), (0, 16, 8), (0, 0, 2), (4, 0, 0)])
@pytest.mark.parametrize("M,N,K", [(70, 130, 200), (700, 512, 256), (5, 64, 1000)])
def test_strides_and_alignment(M, N, K, kind, pad, shift, out_pad):
    check(M, N, K, kind, "bf16", True, "none", pad, shift, out_pad)
    check(M, N, K, kind, "fp32", False, "none", pad, shift, out_pad)


@pytest.mark.parametrize("M,N", [(3, 5), (300, 512), (4000, 640), (20000, 1032)])  # every kernel
def test_no_sum(M, N):
    """K = 0: the activation of the bias."""
    bias = torch.linspace(-2, 2, N, device="cuda")
    out = torch.full((M, N), 5.0, device="cuda")
    e = torch.empty(M, 0, dtype=torch.int8, device="cuda"), torch.empty(N, 0, dtype=torch.int8, device="cuda")
    one = torch.ones(max(M, N), device="cuda")
    pdx.matmul8(e[0], one[:M], e[1], one[:N], out, bias=bias, act="relu")
    torch.cuda.synchronize()
    assert torch.equal(out, bias.clamp(min=0).expand(M, N))


def test_int8_sums_are_exact():
    """Sums past 2^24, with all codes at their ends."""
    M, N, K = 130, 70, 4111
    a = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), 127, dtype=torch.int8, device="cuda")
    w[1] = -128
    out = torch.empty(M, N, device="cuda")
    pdx.matmul8(a, torch.ones(M, device="cuda"), w, torch.ones(N, device="cuda"), out)
    torch.cuda.synchronize()
    assert torch.all(out[:, 1] == float(128 * 128 * K)) and torch.all(out[:, 0] == torch.tensor(float(-128 * 127 * K)).item())


@pytest.mark.parametrize("M", [4, 300])
def test_scales_and_codes_that_are_not_finite(M):
    """A NaN scale or code marks its own row or column and no other."""
    g = tc.gen(4)
    a, w = codes(g, M, 64, "e4m3").clone(), codes(g, 96, 64, "e4m3").clone()
    a.view(torch.uint8)[2, 5] = 0x7f  # NaN
    sa, sw = torch.ones(M, device="cuda"), torch.ones(96, device="cuda")
    sa[1] = float("nan")
    sw[3] = float("inf")
    out = torch.empty(M, 96, dtype=torch.bfloat16, device="cuda")
    pdx.matmul8(a, sa, w, sw, out)
    torch.cuda.synchronize()
    bad = ~torch.isfinite(out)
    assert bad[1].all() and bad[2].all() and bad[:, 3].all()
    rest = torch.ones_like(bad)
    rest[1:3] = False
    rest[:, 3] = False
    assert not bad[rest].any()


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("M,N,K", [(180, 512, 512), (3000, 512, 512), (300, 333, 777)])
def test_same_bits_again_and_on_another_stream(M, N, K, kind):
    g = tc.gen(8)
    a, w = codes(g, M, K, kind), codes(g, N, K, kind)
    sa, sw = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    outs = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pdx.matmul8(a, sa, w, sw, outs[0])
    pdx.matmul8(a, sa, w, sw, outs[1])
    pdx.matmul8(a, sa, w, sw, outs[2], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_refusals():
    a = torch.zeros(4, 32, dtype=torch.int8, device="cuda")
    w = torch.zeros(8, 32, dtype=torch.int8, device="cuda")
    sa, sw, out = torch.ones(4, device="cuda"), torch.ones(8, device="cuda"), torch.empty(4, 8, device="cuda")
    for bad in (dict(w=w.view(torch.float8_e4m3fn)), dict(w=w[:, :16]), dict(a=a.view(torch.uint8)), dict(out=out.half()), dict(out=out[:3]),
                dict(a_scales=sa[:3]), dict(w_scales=sw.double()), dict(bias=sa), dict(a=a.cpu()), dict(w=w.cpu()),
                dict(out=torch.empty(8, 4, device="cuda").t())):
        with pytest.raises((ValueError, pdx.PredecoderError)):
            pdx.matmul8(**(dict(a=a, a_scales=sa, w=w, w_scales=sw, out=out) | bad))
    with pytest.raises(pdx.PredecoderError) as e:
        pdx.matmul8(a, sa, w, sw, out, act=7)
    assert e.value.status == pdx.PD_ERR_INVALID_ARG
    K = 133145
    with pytest.raises(pdx.PredecoderError) as e:
        pdx.matmul8(torch.zeros(1, K, dtype=torch.int8, device="cuda"), sa[:1], torch.zeros(1, K, dtype=torch.int8, device="cuda"), sw[:1],
                    out[:1, :1])
    assert e.value.status == pdx.PD_ERR_UNSUPPORTED


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_results_larger_than_the_caches(kind, out):
    """Results that are stored past the caches are those of the rows one part at a time (sums do not depend on the tile
    that a row is in: exact, or k by k in order)."""
    M, N, K = 70000, 1032, 256
    g = tc.gen(2)
    a, w = codes(g, M, K, kind), codes(g, N, K, kind)
    sa, sw, b = torch.rand(M, device="cuda"), torch.rand(N, device="cuda") / 1000, tc.normal(g, N)
    whole = torch.empty(M, N, dtype=tc.DTYPES[out], device="cuda")
    pdx.matmul8(a, sa, w, sw, whole, bias=b, act="gelu")
    part = torch.empty(1000, N, dtype=tc.DTYPES[out], device="cuda")
    for lo in (0, 33000, 69000):
        pdx.matmul8(a[lo:lo + 1000], sa[lo:lo + 1000], w, sw, part, bias=b, act="gelu")
        torch.cuda.synchronize()
        want, size = tc.matmul64(a[lo:lo + 1000], sa[lo:lo + 1000], w, sw, b, "gelu")
        for o in (part, whole[lo:lo + 1000]):
            assert torch.all((o.double() - want).abs() <= tc.matmul_tolerance(want, size, b, kind == "int8", o.dtype, K))
        if kind == "int8":
            assert torch.equal(part, whole[lo:lo + 1000])
