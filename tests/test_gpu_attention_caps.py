"""GPU: attention whose scores are capped far outside the usual range, against its definition in 64 bits.

The score's error is bounded by its own size, not by the cap's: D roundings of the product, and 24 of the capped score (cap,
argument, exponential, reciprocal and their sum give 19 relative to it, the reference that it is taken from and the sum
with it the rest)."""
import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu


def qkv(g, B, nq, nk, H, Hk, D, spread):
    q = (spread * tc.normal(g, B, nq, H, D)).to(torch.bfloat16)
    kv = tc.normal(g, B, nk, 2, Hk, D).to(torch.bfloat16)
    return q, kv[:, :, 0], kv[:, :, 1]


def check(q, k, v, sites=None, cap=0.0, slopes=None, causal=False, scale=None):
    B, nq, H, D = q.shape
    out = torch.full_like(q, 9.0)
    pdx.attention(q, k, v, out, sites, sites, scale=scale, cap=cap, slopes=slopes, causal=causal)
    torch.cuda.synchronize()
    s = D ** -0.5 if scale is None else scale
    want, moved, _ = tc.attention64(q, k, v, sites, sites, s, cap, slopes, causal, 0)
    a, b = q.double().transpose(1, 2), k.double().transpose(1, 2).repeat_interleave(H // k.shape[2], 1)
    size = float((a.abs() @ b.abs().transpose(2, 3).contiguous()).amax()) * abs(s)
    most = float((a @ b.transpose(2, 3).contiguous()).abs().amax()) * abs(s)
    far = 0.0
    if slopes is not None:
        far = float(slopes.max()) * float((sites[:, None, :3] - sites[None, :, :3]).abs().sum(-1).max())
    score = D * tc.U32 * size + 24 * tc.U32 * min(most, cap) + 4 * tc.U32 * far
    assert torch.all((out.double() - want).abs() <= tc.attention_tolerance(want, moved, score))
    return out


@pytest.mark.parametrize("cap", [64.5, 300.0, 1e4, 1e6, 1e8, 1e30, 3.4e38])
@pytest.mark.parametrize("spread", [1.5, 60.0])
@pytest.mark.parametrize("nq,nk,D", [(1, 63, 64), (40, 129, 64), (150, 200, 128), (300, 700, 32)])
def test_large_caps(cap, spread, nq, nk, D):
    """Whole tiles, ends inside a tile, one token and many."""
    g = tc.gen(nq + nk)
    check(*qkv(g, 2, nq, nk, 2, 1, D, spread), cap=cap)


@pytest.mark.parametrize("cap", [1e4, 1e6, 1e30])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("shapes", [((5, 5), (3, 7)), ((3, 2), (5, 9), (3, 1), (7, 6))])
def test_large_caps_where_tiles_are_masked(cap, causal, bias, shapes):
    """Volumes that meet inside tiles, rounds up to a row's own, with and without notes of the tiles."""
    g = tc.gen(len(shapes))
    sites = torch.cat([pdx.volume_sites(d, T, n) for n, (d, T) in enumerate(shapes)])
    n = sites.shape[0]
    slopes = torch.tensor([0.25, 0.05], device="cuda") if bias else None
    check(*qkv(g, 1, n, n, 2, 1, 64, 1.5), sites, cap=cap, slopes=slopes, causal=causal)


@pytest.mark.parametrize("nk", [64, 200])
def test_scores_past_a_large_cap(nk):
    """Scores around and beyond the cap are capped, with the cap's own precision."""
    g = tc.gen(nk)
    q, k, v = qkv(g, 1, 70, nk, 2, 2, 64, 1.5)
    check(q, k, v, cap=100.0, scale=20.0)
    check(q, k, v, cap=100.0, scale=-4.0)


@pytest.mark.parametrize("cap,scale", [(1e-39, 1.0), (1e-30, 1e20), (0.0, 3e38), (50.0, 3e38), (100.0, 3e38)])
@pytest.mark.parametrize("nk", [64, 130])
def test_scores_of_zero_where_scale_and_cap_leave_the_range(cap, scale, nk):
    """Scores of zero stay zero though scale / cap, or the scale in the softmax's units, is past the largest number."""
    g = tc.gen(nk + 1)
    q, k, v = qkv(g, 1, 70, nk, 2, 1, 64, 0.0)
    assert torch.isfinite(check(q, k, v, cap=cap, scale=scale)).all()


@pytest.mark.parametrize("cap", [30.0, 1e4])
@pytest.mark.parametrize("nk", [64, 130])
def test_products_whose_square_leaves_the_range(cap, nk):
    """Usual scores of huge products and a tiny scale."""
    g = tc.gen(nk + 2)
    q, k, v = qkv(g, 1, 70, nk, 2, 1, 64, 1e10)
    check(q, (1e10 * k.float()).to(torch.bfloat16), v, cap=cap, scale=2.0 ** -70)


@pytest.mark.parametrize("slope", [1e32, 3.4e38])
@pytest.mark.parametrize("cap", [0.0, 30.0, 1e4])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,T", [(5, 5), (7, 9)])
def test_slopes_that_leave_the_nearest_token(slope, cap, causal, d, T):
    """A finite slope of any size times a distance of zero is zero: every token sees itself alone."""
    g = tc.gen(d)
    sites = pdx.volume_sites(d, T)
    n = sites.shape[0]
    q, k, v = qkv(g, 1, n, n, 2, 2, 64, 1.5)
    out = torch.full_like(q, 9.0)
    pdx.attention(q, k, v, out, sites, sites, cap=cap, slopes=torch.full((2,), slope, device="cuda"), causal=causal)
    torch.cuda.synchronize()
    assert torch.equal(out, v)
