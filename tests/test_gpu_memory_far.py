"""GPU: what a stream keeps, where offsets pass 32 bits: a cache of 8.6 GB, rows that lie far apart."""
import pytest
import torch

import memory_cases as mc
import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu

FREE = 40 << 30  # bytes that the largest test asks for, and some


def need_memory():
    if torch.cuda.mem_get_info()[0] < FREE:
        pytest.skip("less than 40 GiB of free memory on the GPU")


def sites_of(B, n):
    s = torch.zeros(B, n, 4, dtype=torch.int32, device="cuda")
    s[..., 0] = torch.arange(n, device="cuda") // 4
    s[..., 1] = torch.arange(n, device="cuda") % 4
    return s


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
def test_long_cache(codes):
    """Tokens over the end of a ring of 33.7 million places: written, read and attended to as in a ring that just holds them."""
    need_memory()
    capacity, n, D, H = 33_700_000, 300, 128, 2
    g = tc.gen(41)
    k, v = tc.normal(g, 1, n, 1, D), tc.normal(g, 1, n, 1, D)
    sites = sites_of(1, n)
    big, small = pdx.new_cache(1, capacity, 1, D, codes), pdx.new_cache(1, n, 1, D, codes)
    assert big[0].numel() > 1 << 32
    at = torch.tensor([capacity - 200], device="cuda")
    pdx.cache_write(big, at, k, v, sites)
    pdx.cache_write(small, at * 0, k, v, sites)
    index = mc.places(at, n, capacity)[0]
    assert torch.equal(big[0].view(torch.int8)[:, :, :, index], small[0].view(torch.int8))
    assert torch.equal(big[1][:, :, :, index], small[1]) and torch.equal(big[2][:, index], small[2])
    assert int((big[2][..., 3] >= 0).sum()) == n
    got = [torch.empty_like(k) for _ in range(4)]
    pdx.cache_read(big, at, got[0], got[1])
    pdx.cache_read(small, at * 0, got[2], got[3])
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])
    for m in (1, 100):
        q = tc.normal(g, 1, m, H, D).to(torch.bfloat16)
        a = dict(scale=D ** -0.5, cap=20.0, slopes=torch.tensor([0.1, 0.5], device="cuda"), causal=True, prefix=None)
        out = torch.empty_like(q)
        pdx.attention8(q, big, out, sites[:, n - m:], **a)
        want, bound = mc.attention8_reference(q, small, sites[:, n - m:], **(a | dict(prefix=-(1 << 31))))
        assert torch.all((out.double() - want).abs() <= bound)


@pytest.mark.parametrize("n,per_round", [(120, 40), (120, 3), (1, 1)])
def test_linear_rows_far_apart(n, per_round):
    """Tokens 2^25 numbers apart, or entries 2^32: results as of tensors without gaps."""
    need_memory()
    H, Hk, D, B = 4, 2, 64, 2
    g = tc.gen(42)
    x = tc.normal(g, B, n, 2 * H + 2 * Hk, D).to(torch.bfloat16)
    slopes = torch.tensor([0.01, 0.3], device="cuda")
    want, want_state = torch.empty(B, n, H, D, device="cuda", dtype=torch.bfloat16), torch.empty(B, Hk, D, D, device="cuda")
    pdx.linear_attention(x[:, :, :H], x[:, :, H:H + Hk], x[:, :, H + Hk:H + 2 * Hk], want, slopes=slopes, per_round=per_round, state_out=want_state)
    width = x.shape[2] * D
    far = torch.empty((1 << 32) + (n << 25) + width, device="cuda", dtype=torch.bfloat16)
    y = far.as_strided(x.shape, (1 << 32 if n == 1 else 1 << 24, 1 << 25, D, 1))
    y.copy_(x)
    out, state = y[:, :, H + 2 * Hk:], torch.empty_like(want_state)
    pdx.linear_attention(y[:, :, :H], y[:, :, H:H + Hk], y[:, :, H + Hk:H + 2 * Hk], out, slopes=slopes, per_round=per_round, state_out=state)
    assert torch.equal(out, want) and torch.equal(state, want_state)


def test_attention8_rows_far_apart():
    need_memory()
    H, Hk, D, n, B = 2, 1, 64, 130, 2
    g = tc.gen(43)
    k, v = tc.normal(g, B, 500, Hk, D), tc.normal(g, B, 500, Hk, D)
    cache = pdx.new_cache(B, 500, Hk, D)
    pdx.cache_write(cache, torch.zeros(B, dtype=torch.int64, device="cuda"), k, v, sites_of(B, 500))
    x = tc.normal(g, B, n, H, D).to(torch.bfloat16)
    far = torch.empty((n << 25) + (1 << 25), device="cuda", dtype=torch.bfloat16)
    for m in (4, n):
        want = torch.empty(B, m, H, D, device="cuda", dtype=torch.bfloat16)
        pdx.attention8(x[:, :m], cache, want, sites_of(B, m), causal=True)
        stride = (n << 25) // m  # tokens; entries half as far
        y = far.as_strided((B, m, 2 * H, D), (stride // 2, stride, D, 1))
        y[:, :, :H] = x[:, :m]
        pdx.attention8(y[:, :, :H], cache, y[:, :, H:], sites_of(B, m), causal=True)
        assert torch.equal(y[:, :, H:], want)


def test_cache_rows_far_apart():
    need_memory()
    Hk, D, n = 2, 32, 130
    g = tc.gen(44)
    x = tc.normal(g, 1, n, 2 * Hk, D).to(torch.bfloat16)
    far = torch.empty(n << 25, device="cuda", dtype=torch.bfloat16)
    y = far.as_strided(x.shape, (0, 1 << 25, D, 1))
    y.copy_(x)
    near, cache, at = pdx.new_cache(1, n, Hk, D), pdx.new_cache(1, n, Hk, D), torch.zeros(1, dtype=torch.int64, device="cuda")
    pdx.cache_write(near, at, x[:, :, :Hk], x[:, :, Hk:], sites_of(1, n))
    pdx.cache_write(cache, at, y[:, :, :Hk], y[:, :, Hk:], sites_of(1, n))
    assert all(torch.equal(a.view(torch.int8), b.view(torch.int8)) for a, b in zip(near, cache))
    z = torch.empty_like(x)
    pdx.cache_read(cache, at, z[:, :, :Hk], z[:, :, Hk:])
    y.zero_()
    pdx.cache_read(cache, at, y[:, :, :Hk], y[:, :, Hk:])
    assert torch.equal(y, z)
