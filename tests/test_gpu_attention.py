"""GPU: attention over the tokens of detector volumes against its definition in 64 bits."""
import math

import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu


def qkv(g, B, nq, nk, H, Hk, D, spread=1.5):
    q = (spread * tc.normal(g, B, nq, H, D)).to(torch.bfloat16)
    kv = tc.normal(g, B, nk, 2, Hk, D).to(torch.bfloat16)
    return q, kv[:, :, 0], kv[:, :, 1]


def slopes_of(H):
    return torch.exp2(-4.0 * (torch.arange(H, device="cuda") + 1.0) / H)


def check(q, k, v, q_sites=None, k_sites=None, cap=0.0, slopes=None, causal=False, prefix=0, scale=None, out=None):
    B, nq, H, D = q.shape
    if out is None:
        out = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device="cuda")
    pdx.attention(q, k, v, out, q_sites, k_sites, scale=scale, cap=cap, slopes=slopes, causal=causal, prefix=prefix)
    torch.cuda.synchronize()
    s = D ** -0.5 if scale is None else scale
    want, moved, score = tc.attention64(q, k, v, q_sites, k_sites, s, cap, slopes, causal, prefix)
    ok = (out.double() - want).abs() <= tc.attention_tolerance(want, moved, score)
    same = torch.isnan(out) & torch.isnan(want) | (out.double() == want)
    assert torch.all(ok | same)
    return out, want


def volumes(*shapes):
    return torch.cat([pdx.volume_sites(d, T, n) for n, (d, T) in enumerate(shapes)])


# one token, sizes around the tiles of queries (32, 128) and keys (32, 64), grouped heads, every head width
@pytest.mark.parametrize("B,nq,nk,H,Hk,D", [(1, 1, 1, 1, 1, 8), (2, 1, 64, 4, 1, 32), (1, 3, 65, 6, 2, 64), (3, 33, 31, 2, 2, 48), (1, 128, 128, 2, 1, 128),
                                            (2, 129, 200, 3, 3, 64), (1, 300, 1, 2, 2, 32), (1, 7, 1500, 8, 2, 64), (2, 190, 333, 4, 4, 96),
                                            (1, 64, 63, 1, 1, 16), (1, 1, 5000, 2, 1, 128), (4, 2, 700, 64, 1, 24), (1, 513, 640, 2, 2, 104)])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_every_token_seen(B, nq, nk, H, Hk, D, cap):
    g = tc.gen(B + nq * 3 + nk * 5 + D)
    check(*qkv(g, B, nq, nk, H, Hk, D), cap=cap)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("causal,prefix", [(False, 0), (True, 0), (True, 2)])
def test_volumes_packed_in_one_row(D, cap, bias, causal, prefix):
    g = tc.gen(D + int(cap))
    sites = volumes((3, 2), (5, 5), (3, 1), (7, 9), (5, 3), (3, 7))
    n = sites.shape[0]
    check(*qkv(g, 1, n, n, 4, 2, D), sites, sites, cap=cap, slopes=slopes_of(4) if bias else None, causal=causal, prefix=prefix)


@pytest.mark.parametrize("causal", [False, True])
def test_tokens_in_any_order(causal):
    """Volumes and rounds shuffled over the row: the masks go by the sites, not by the order."""
    g = tc.gen(6)
    sites = volumes((5, 6), (7, 5), (3, 9))
    a = sites[torch.randperm(sites.shape[0], generator=g, device="cuda")].contiguous()
    b = sites[torch.randperm(sites.shape[0], generator=g, device="cuda")].contiguous()
    n = sites.shape[0]
    check(*qkv(g, 1, n, n, 2, 1, 64), a, b, cap=15.0, slopes=slopes_of(2), causal=causal, prefix=1 if causal else 0)


def test_a_list_of_sites_for_each_entry():
    g = tc.gen(7)
    sites = torch.stack([pdx.volume_sites(5, 9, 0), pdx.volume_sites(5, 9, 3, first_round=40), volumes((5, 2), (5, 7))])
    n = sites.shape[1]
    check(*qkv(g, 3, n, n, 4, 1, 32), sites, sites, slopes=slopes_of(4), causal=True)


@pytest.mark.parametrize("far", [0, 1 << 20, -(1 << 20), (1 << 29) - 600])
@pytest.mark.parametrize("axis", [0, 1, 2])
def test_far_coordinates(far, axis):
    """Coordinates beyond a byte, beyond 16 bits, negative ones: distances stay exact."""
    g = tc.gen(8)
    sites = pdx.volume_sites(7, 8)
    sites[:, axis] += far
    sites[::5, axis] -= 300
    n = sites.shape[0]
    check(*qkv(g, 1, n, n, 2, 2, 32), sites, sites, slopes=slopes_of(2) / 8, causal=axis == 0)


@pytest.mark.parametrize("new", [1, 5, 36])
@pytest.mark.parametrize("H,Hk", [(8, 2), (3, 3), (64, 1)])
def test_new_tokens_against_caches_of_unequal_length(new, H, Hk):
    g = tc.gen(new)
    B, rounds = 3, 60
    sites = pdx.volume_sites(5, rounds).repeat(B, 1, 1)
    lengths = [60, 1, 37]
    for b, n in enumerate(lengths):
        sites[b, :, 3] = torch.where(sites[b, :, 0] < n, b, -1)
    q_sites = torch.stack([sites[b, (n - 1) * 36:(n - 1) * 36 + new] for b, n in enumerate(lengths)])
    q, k, v = qkv(g, B, new, rounds * 36, H, Hk, 64)
    for b, n in enumerate(lengths):  # what an unused cache may hold
        k[b, n * 36:] = float("nan")
        v[b, n * 36:] = float("inf")
    out, _ = check(q, k, v, q_sites, sites, cap=30.0, slopes=slopes_of(H), causal=True)
    assert torch.isfinite(out).all()


def test_rows_that_see_nothing():
    g = tc.gen(10)
    sites = volumes((3, 4), (5, 4))
    n = sites.shape[0]
    q_sites = sites.clone()
    q_sites[::3, 3] = -1   # no token
    q_sites[1::3, 3] = 77  # a volume without keys
    q, k, v = qkv(g, 1, n, n, 2, 1, 64)
    out, _ = check(q, k, v, q_sites, sites)
    assert torch.all(out[:, ::3] == 0) and torch.all(out[:, 1::3] == 0)
    k[:] = float("nan")
    v[:] = float("nan")
    pdx.attention(q, k, v, out, torch.full_like(q_sites, -1), sites)
    torch.cuda.synchronize()
    assert torch.all(out == 0)
    pdx.attention(q, k[:, :0], v[:, :0], out.fill_(3.0), q_sites, sites[:0])  # no keys at all
    torch.cuda.synchronize()
    assert torch.all(out == 0)
    pdx.attention(q, k[:, :0], v[:, :0], out.fill_(3.0))
    torch.cuda.synchronize()
    assert torch.all(out == 0)


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan"), 3.3e38])
@pytest.mark.parametrize("causal", [False, True])
def test_odd_values_in_some_keys(value, causal):
    """Infinities and NaN in single values and keys reach the rows that see them, and no others."""
    g = tc.gen(12)
    sites = volumes((3, 6), (3, 6), (3, 6))
    n = sites.shape[0]
    q, k, v = qkv(g, 1, n, n, 2, 1, 64)
    # one key of volume 0, and the last round of volume 2 (rows before it do not see it when causal)
    v[0, 20, 0, 3] = value
    v[0, n - 1, 0, 7] = value
    out, want = check(q, k, v, sites, sites, causal=causal)
    assert torch.isfinite(out[0, 96:192]).all()
    if causal and value != 3.3e38:
        assert not torch.isfinite(out[0, 192 + 80:, :, 7]).any() and torch.isfinite(out[0, 192:192 + 80]).all()
    if value != 3.3e38:
        assert torch.equal(torch.isfinite(out), torch.isfinite(want))
        v[0, 20, 0, 3] = v[0, n - 1, 0, 7] = 0.0
        k[0, n - 1] = value  # scores that are not finite
        out, _ = check(q[:, :192], k, v, sites[:192].contiguous(), sites, causal=causal)
        assert torch.isfinite(out).all()


@pytest.mark.parametrize("cap", [0.0, 40.0])
@pytest.mark.parametrize("spread", [0.0, 30.0, 200.0])
def test_scores_of_any_size(cap, spread):
    """Equal scores; scores that leave one key; scores in the thousands, far below zero for whole tiles before they rise."""
    g = tc.gen(13)
    q, k, v = qkv(g, 1, 200, 500, 2, 2, 64, spread)
    check(q, k, v, cap=cap)
    k[:, :400] *= torch.linspace(0, 1, 400, device="cuda").to(torch.bfloat16)[None, :, None, None]
    check(q, k, v, cap=cap)
    sites = pdx.volume_sites(9, 5)
    check(q, k, v, sites[:200].contiguous(), sites, cap=cap, slopes=torch.tensor([50.0, 1000.0], device="cuda"))
    check(q, k, v, sites[:200].contiguous(), sites, cap=cap, slopes=torch.tensor([-0.5, 0.25], device="cuda"))
    check(q, k, v, cap=cap, scale=-0.3)


def test_strides():
    """Rows of a joint projection, a cache with keys and values side by side, heads before tokens, padded entries."""
    g = tc.gen(14)
    B, n, H, Hk, D = 2, 150, 4, 2, 64
    joint = tc.normal(g, B, n, H + 2 * Hk + 1, D).to(torch.bfloat16)
    out = torch.full((B, n + 3, H + 1, D), 4.0, dtype=torch.bfloat16, device="cuda")
    check(joint[:, :, :H], joint[:, :, H:H + Hk], joint[:, :, H + Hk:H + 2 * Hk], out=out[:, :n, :H])
    assert torch.all(out[:, n:] == 4.0) and torch.all(out[:, :, H:] == 4.0)
    q, k, v = (tc.normal(g, B, h, n, D).to(torch.bfloat16).transpose(1, 2) for h in (H, Hk, Hk))
    check(q, k, v, out=torch.empty(B, H, n, D, dtype=torch.bfloat16, device="cuda").transpose(1, 2))
    check(q.expand(B, n, H, D), k[:1].expand(B, n, Hk, D), v[:1].expand(B, n, Hk, D))


def test_offsets_past_32_bits():
    """Tokens of a cache that lie more than 2^32 bytes apart."""
    g = tc.gen(15)
    n, D = 130, 64
    step = (1 << 32) // (2 * 128) + 8  # values from token to token: 130 of them span 4.4 GB
    step -= step % 8
    whole = torch.zeros(2 * n * step, dtype=torch.bfloat16, device="cuda")
    kv = whole.view(2, n, 1, step)[..., :D]
    kv.copy_(tc.normal(g, 2, n, 1, D))
    q = tc.normal(g, 1, 40, 2, D).to(torch.bfloat16)
    check(q, kv[:1], kv[1:])
    del whole, kv
    torch.cuda.empty_cache()


@pytest.mark.parametrize("nq,nk", [(300, 700), (1, 6000)])
def test_same_bits_again_on_another_stream_and_in_a_graph(nq, nk):
    g = tc.gen(16)
    q, k, v = qkv(g, 2, nq, nk, 8, 2, 64)
    sites = pdx.volume_sites(13, 40)[:nk].contiguous()
    a = dict(q_sites=sites[:nq].contiguous(), k_sites=sites, cap=30.0, slopes=slopes_of(8), causal=True)
    first, again, there, played = (torch.zeros_like(q) for _ in range(4))
    pdx.attention(q, k, v, first, **a)
    pdx.attention(q, k, v, again, **a)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pdx.attention(q, k, v, there, stream=s, **a)
    torch.cuda.synchronize()
    assert torch.equal(first, again) and torch.equal(first, there)
    ws = torch.empty(max(16, pdx.attention_workspace(q, k, v, played, **a)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pdx.attention(q, k, v, played, workspace=ws, **a)
    for n in range(3):
        q.copy_(tc.normal(tc.gen(n), *q.shape).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        pdx.attention(q, k, v, first, **a)
        torch.cuda.synchronize()
        assert torch.equal(first, played)


def test_refusals():
    q = torch.zeros(1, 4, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(1, 9, 2, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    sites = torch.zeros(9, 4, dtype=torch.int32, device="cuda")
    good = dict(q=q, k=k, v=k, out=out)
    for bad in (dict(v=k[:, :8]), dict(k=k.float()), dict(out=out[:, :3]), dict(q=q[0]), dict(q_sites=sites[:4]), dict(k_sites=sites),
                dict(q_sites=sites[:3], k_sites=sites), dict(q_sites=sites[:4].long(), k_sites=sites), dict(k=k.cpu()),
                dict(q_sites=sites[:4], k_sites=sites, slopes=torch.zeros(3, device="cuda")),
                dict(q=q.transpose(2, 3).contiguous().transpose(2, 3))):
        with pytest.raises(ValueError):
            pdx.attention(**(good | bad))
    s = dict(q_sites=sites[:4], k_sites=sites)
    three = torch.zeros(1, 9, 3, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(causal=True), dict(slopes=torch.zeros(4, device="cuda")), s | dict(prefix=2), s | dict(causal=True, prefix=-1), dict(cap=-1.0),
                dict(scale=math.nan), dict(cap=math.inf), dict(k=three, v=three)):
        with pytest.raises(pdx.PredecoderError) as e:
            pdx.attention(**(good | bad))
        assert e.value.status == pdx.PD_ERR_INVALID_ARG
    wide = torch.zeros(1, 4, 4, 136, dtype=torch.bfloat16, device="cuda")
    odd = torch.zeros(1, 4, 4, 12, dtype=torch.bfloat16, device="cuda")
    for t in (wide, odd, wide[..., 4:132], wide[..., :64].as_strided((1, 4, 4, 64), (0, 260, 65, 1))):
        with pytest.raises(pdx.PredecoderError) as e:
            pdx.attention(t, t, t, torch.empty_like(t, memory_format=torch.contiguous_format))
        assert e.value.status == pdx.PD_ERR_UNSUPPORTED


def test_scores_of_zero_under_a_tiny_cap():
    """scale / cap so large that the small scores' polynomial has no coefficients: scores of zero are zero all the same."""
    g = tc.gen(18)
    q, k, v = qkv(g, 1, 70, 130, 2, 1, 64)
    out, _ = check(torch.zeros_like(q), k, v, cap=1e-8, scale=1.0)
    assert torch.isfinite(out).all()
