"""GPU: keys and values into a ring of places in 8 bits and back, against 64 bits."""
import math

import pytest
import torch

import memory_cases as mc
import paper_2604_12841_amd as pdx
import token_cases as tc
from memory_cases import CODES

pytestmark = pytest.mark.gpu


def sites_of(g, B, n, holes):
    s = torch.randint(-50, 50, (B, n, 4), generator=g, device="cuda", dtype=torch.int32)
    s[..., 3] = torch.arange(B, device="cuda", dtype=torch.int32)[:, None]
    if holes:
        s[..., 3] = torch.where(torch.rand(B, n, generator=g, device="cuda") < 0.3, -1 - s[..., 3], s[..., 3])
    return s


def expected_write(cache, at, k, v, sites):
    """The cache after the write, codes in 64 bits."""
    codes, scales, kept = cache[0].double(), cache[1].clone(), cache[2].clone()
    place = mc.places(at, k.shape[1], kept.shape[1])
    for b in range(k.shape[0]):
        on = (sites[b, :, 3] >= 0).nonzero().flatten()
        p = place[b, on]
        kept[b, p] = sites[b, on]
        for n, x in enumerate((k, v)):
            y, s = mc.quantise64(x[b, on].transpose(0, 1), cache[0].dtype)
            codes[b, n][:, p], scales[b, n][:, p] = y, s
    return codes, scales, kept


def same(a, b):
    return torch.equal(a.nan_to_num(nan=12345.0), b.nan_to_num(nan=12345.0))


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,n,capacity,Hk,D", [(1, 1, 1, 1, 16), (1, 1, 7, 3, 32), (2, 36, 36, 4, 32), (3, 131, 260, 2, 64), (2, 65, 196, 5, 48),
                                               (1, 300, 301, 1, 128), (5, 17, 64, 3, 96), (2, 40, 50, 2, 80), (1, 9, 9, 2, 112)])
def test_write_and_read(codes, dtype, B, n, capacity, Hk, D):
    g = tc.gen(n * 100 + D)
    dt = tc.DTYPES[dtype]
    old = torch.full((B, capacity, 4), 5, dtype=torch.int32, device="cuda")
    cache = mc.filled_cache(g, B, capacity, Hk, D, codes, old)
    k, v = ((tc.normal(g, B, n, Hk, D) * torch.exp(2.0 * tc.normal(g, B, n, Hk, 1))).to(dt) for _ in range(2))
    k[0, 0, 0] = 0.0
    v[0, n // 2, Hk - 1, 3] = math.inf
    v[B - 1, n - 1, 0, D - 1] = math.nan
    sites = sites_of(g, B, n, holes=True)
    at = torch.randint(-3 * capacity, 3 * capacity, (B,), generator=g, device="cuda")
    at[0] = capacity - 1
    at[B - 1] = (1 << 62) + 11
    want = expected_write(cache, at, k, v, sites)
    pdx.cache_write(cache, at, k, v, sites)
    torch.cuda.synchronize()
    assert torch.equal(cache[0].double(), want[0])  # codes, and the places that are not written
    assert same(cache[1], want[1]) and torch.equal(cache[2], want[2])
    # back: one product (rounded to fp32) and the type's rounding
    for out_type in (torch.bfloat16, torch.float32):
        a, b = (torch.full((B, n, Hk, D), 9.0, device="cuda", dtype=out_type) for _ in range(2))
        back = torch.empty(B, n, 4, dtype=torch.int32, device="cuda")
        pdx.cache_read(cache, at, a, b, back)
        torch.cuda.synchronize()
        place = mc.places(at, n, capacity)
        rows = torch.arange(B, device="cuda")[:, None]
        assert torch.equal(back, cache[2][rows, place])
        on = (back[..., 3] >= 0)[..., None, None]
        for got, whole in zip((a, b), mc.by_token(cache)):
            ref = torch.where(on, whole[rows, place], 0.0)
            assert torch.equal(got.isnan(), ref.isnan())
            got, ref = got.double().nan_to_num(0), ref.nan_to_num(0)
            assert torch.all((got - ref).abs() <= (tc.U32 + (tc.U16 if out_type == torch.bfloat16 else 0)) * ref.abs() + 1e-45)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_values_at_the_borders(codes, dtype):
    """Middles between two codes, neighbours of middles, rows of the smallest and largest numbers."""
    D, dt = 128, tc.DTYPES[dtype]
    q = mc.QMAX[CODES[codes]]
    rows = []
    for top in (q, 3.0, 254.0, 7.0, 1.0, 2.0 ** -126, 2.0 ** -140, 127 * 2.0 ** -149, 2.0 ** -149, 2.0 ** 127, 3.3e38, 2.0 ** -60, 1.5 * 2.0 ** -61):
        scale = top / q
        m = torch.arange(D, dtype=torch.float64)
        mid = (m + 0.5) * scale if codes == "int8" else ((16 + m % 16 + 0.5) / 16) * 2.0 ** (m // 16) * scale
        x = mid.clamp(max=top)
        x[0] = top
        rows += [x, -x, x * (1 + 2.0 ** -23), x * (1 - 2.0 ** -24), x.flip(0) / 3, x * x / top]
    x = torch.stack(rows).clamp(-3.38e38, 3.38e38).to(torch.float32).to(dt).cuda()
    n = x.shape[0]
    x = x.view(1, n, 1, D)
    cache = pdx.new_cache(1, n, 1, D, codes)
    at = torch.zeros(1, dtype=torch.int64, device="cuda")
    sites = torch.zeros(n, 4, dtype=torch.int32, device="cuda")
    pdx.cache_write(cache, at, x, -x, sites)
    torch.cuda.synchronize()
    y, s = mc.quantise64(x[0, :, 0], CODES[codes])
    assert torch.equal(cache[1][0, 0, 0], s) and torch.equal(cache[1][0, 1, 0], s)
    assert torch.equal(cache[0][0, 0, 0].double(), y) and torch.equal(cache[0][0, 1, 0].double(), -y)


@pytest.mark.parametrize("shift,pad", [(0, 2), (1, 0), (3, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("codes", ["e4m3", "int8"])
def test_rows_of_wider_tensors(shift, pad, dtype, codes):
    g = tc.gen(shift * 10 + pad)
    dt, B, n, Hk, D = tc.DTYPES[dtype], 2, 33, 3, 48
    wide = Hk * (2 + pad)
    whole = tc.normal(g, B * n * wide * D + shift).to(dt)
    x = whole[shift:].view(B, n, wide, D)
    k, v = x[:, :, :Hk], x[:, :, Hk:2 * Hk]
    cache = pdx.new_cache(B, 40, Hk, D, codes)
    at = torch.tensor([39, 5], device="cuda")
    sites = sites_of(g, B, n, holes=False)
    want = expected_write(cache, at, k, v, sites)
    pdx.cache_write(cache, at, k, v, sites)
    kept = whole.clone()
    pdx.cache_read(cache, at, k, v)
    torch.cuda.synchronize()
    assert torch.equal(cache[0].double(), want[0]) and torch.equal(cache[1], want[1])
    place, rows = mc.places(at, n, 40), torch.arange(B, device="cuda")[:, None]
    for got, ref in zip((k, v), mc.by_token(cache)):
        ref = ref[rows, place]
        assert torch.all((got.double() - ref).abs() <= (tc.U32 + tc.UNIT[dt]) * ref.abs())
    x[:, :, :2 * Hk] = kept[shift:].view(B, n, wide, D)[:, :, :2 * Hk]
    assert torch.equal(whole, kept)  # nothing outside was written


def test_one_list_of_sites_and_another_stream():
    g = tc.gen(4)
    B, n = 3, 50
    k, v = tc.normal(g, B, n, 2, 64), tc.normal(g, B, n, 2, 64)
    sites = sites_of(g, 1, n, holes=True)[0]
    at = torch.tensor([1, 2, 3], device="cuda")
    one, two = pdx.new_cache(B, 64, 2, 64), pdx.new_cache(B, 64, 2, 64)
    pdx.cache_write(one, at, k, v, sites)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pdx.cache_write(two, at, k, v, sites.expand(B, n, 4).contiguous(), stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8) if a.dtype == torch.float8_e4m3fn else a, b.view(torch.uint8) if b.dtype == torch.float8_e4m3fn else b)
               for a, b in zip(one, two))


def test_nothing_to_do():
    cache = pdx.new_cache(2, 8, 2, 32)
    e = torch.empty(2, 0, 2, 32, device="cuda")
    at = torch.zeros(2, dtype=torch.int64, device="cuda")
    pdx.cache_write(cache, at, e, e, torch.empty(2, 0, 4, dtype=torch.int32, device="cuda"))
    pdx.cache_read(cache, at, e, e)
    torch.cuda.synchronize()
    assert torch.all(cache[2][..., 3] == -1)


def test_refusals():
    cache = pdx.new_cache(2, 8, 2, 32)
    k = torch.zeros(2, 4, 2, 32, device="cuda")
    sites = torch.zeros(4, 4, dtype=torch.int32, device="cuda")
    at = torch.zeros(2, dtype=torch.int64, device="cuda")
    good = dict(cache=cache, at=at, k=k, v=k.clone(), sites=sites)
    for bad in (dict(at=at.int()), dict(at=at[:1]), dict(at=at.cpu()), dict(k=k[:1]), dict(k=k.half()), dict(v=k.bfloat16()), dict(k=k[..., :16]),
                dict(sites=sites[:3]), dict(sites=None), dict(sites=sites.long()), dict(k=k.transpose(2, 3)), dict(v=k.cpu()),
                dict(cache=(cache[0], cache[1], cache[2][:1])), dict(cache=(cache[0].float(), cache[1], cache[2])),
                dict(cache=(cache[0], cache[1].double(), cache[2])), dict(cache=(cache[0], cache[1].cpu(), cache[2])),
                dict(cache=(cache[0].transpose(2, 3), cache[1], cache[2])), dict(k=k.clone().requires_grad_())):
        with pytest.raises(ValueError):
            pdx.cache_write(**(good | bad))
    with pytest.raises(pdx.PredecoderError) as e:  # more tokens than places
        pdx.cache_write(cache, at, torch.zeros(2, 9, 2, 32, device="cuda"), torch.zeros(2, 9, 2, 32, device="cuda"),
                        torch.zeros(9, 4, dtype=torch.int32, device="cuda"))
    assert e.value.status == pdx.PD_ERR_INVALID_ARG
    with pytest.raises(pdx.PredecoderError) as e:  # outputs on each other
        pdx.cache_read(cache, at, k, k)
    assert e.value.status == pdx.PD_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        pdx.cache_read(cache, at, k, k.clone(), sites)
    with pytest.raises(ValueError):
        pdx.new_cache(1, 1, 1, 16, "fp4")


def test_codes_that_want_a_gradient_are_refused():
    codes, scales, sites = pdx.new_cache(2, 8, 2, 32)
    q = torch.zeros(2, 4, 2, 32, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        pdx.attention8(q, (codes.requires_grad_(), scales, sites), torch.empty_like(q), torch.zeros(4, 4, dtype=torch.int32, device="cuda"))
