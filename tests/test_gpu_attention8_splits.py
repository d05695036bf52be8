"""GPU: attention over an 8-bit cache in several splits, joined: what far splits hold, and splits that see nothing."""
import math

import pytest
import torch

import memory_cases as mc
import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu

# n_q, capacity, heads, kv_heads, D: few rows; more of them, joined a row a workgroup; rows enough for the join of a row in a few threads, at
# each width that is compiled
CASES = [(1, 4000, 4, 2, 64), (1, 5000, 2, 1, 128), (8, 3000, 4, 2, 32), (40, 4000, 4, 2, 64), (40, 3000, 2, 1, 128), (600, 2500, 4, 2, 32), (300, 2500, 8, 2, 48),
         (600, 2500, 4, 2, 128)]


def stream(codes, n, capacity, H, Hk, D):
    """A cache whose place m holds a token of round m / 8, and queries of the last rounds."""
    g = tc.gen(n + capacity + D)
    sites = torch.zeros(1, capacity, 4, dtype=torch.int32, device="cuda")
    sites[0, :, 0] = torch.arange(capacity, device="cuda") // 8
    q_sites = torch.zeros(1, n, 4, dtype=torch.int32, device="cuda")
    q_sites[..., 0] = capacity // 8 - torch.arange(n, device="cuda") % 3
    return mc.filled_cache(g, 1, capacity, Hk, D, codes, sites), tc.normal(g, 1, n, H, D).to(torch.bfloat16), q_sites


def attend(q, cache, q_sites, slopes):
    """The result and its bound's parts; the workspace holds NaN before the call, so that what no split wrote must not be read."""
    out = torch.empty_like(q)
    need = pdx.attention8_workspace(q, cache, out, q_sites, slopes=slopes)
    assert need > 0  # several splits
    work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    pdx.attention8(q, cache, out, q_sites, slopes=slopes, workspace=work)
    torch.cuda.synchronize()
    want, bound = mc.attention8_reference(q, cache, q_sites, q.shape[-1] ** -0.5, 0.0, slopes, False, -(1 << 31))
    assert torch.equal(out.isnan(), want.isnan())
    assert torch.all(((out.double() - want).abs() <= bound) | want.isnan())
    return out


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("n,capacity,H,Hk,D", CASES)
def test_what_is_not_finite_stays_however_far(codes, n, capacity, H, Hk, D):
    """One scale of a key or of a value is NaN, at a token whose weight is 0 beside the nearest ones (200 log2 units and more below them)."""
    cache, q, q_sites = stream(codes, n, capacity, H, Hk, D)
    slopes = torch.ones(H, device="cuda")
    assert torch.isfinite(attend(q, cache, q_sites, slopes)).all()
    for which in (0, 1):
        kept = cache[1][0, which, 0, 3].clone()
        cache[1][0, which, 0, 3] = math.nan
        out = attend(q, cache, q_sites, slopes)
        assert out[:, :, :H // Hk].isnan().all() and torch.isfinite(out[:, :, H // Hk:]).all()
        cache[1][0, which, 0, 3] = kept


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("n,capacity,H,Hk,D", CASES)
def test_splits_without_a_finite_score(codes, n, capacity, H, Hk, D):
    """All keys of the last 600 places have NaN scales, and the farthest tokens scores past 126 log2 units, by a negative slope."""
    cache, q, q_sites = stream(codes, n, capacity, H, Hk, D)
    cache[1][0, 0, 0, capacity - 600:] = math.nan
    out = attend(q, cache, q_sites, -torch.ones(H, device="cuda"))
    assert out[:, :, :H // Hk].isnan().all() and torch.isfinite(out[:, :, H // Hk:]).all()


@pytest.mark.parametrize("n,capacity,H,Hk,D", CASES)
def test_splits_that_see_nothing(n, capacity, H, Hk, D):
    """Tokens at the ends alone, with scores far apart: the splits between them leave no result, and none is read."""
    cache, q, q_sites = stream("e4m3", n, capacity, H, Hk, D)
    cache[2][:, 100:capacity - 100, 3] = -1
    cache[1][:, :, :, 100:capacity - 100] = math.nan
    for slope in (1.0, 0.01, -1.0):
        assert torch.isfinite(attend(q, cache, q_sites, torch.full((H,), slope, device="cuda"))).all()
