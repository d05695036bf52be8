"""GPU: the scores of attention over an 8-bit cache, in tiles that all rows see whole: each form of the cap by results that are made to cancel,
and the distance's part on both sides of the rounds that are a multiple of 256."""
import math

import pytest
import torch

import memory_cases as mc
import paper_2604_12841_amd as pdx
import token_cases as tc
from memory_cases import CODES
from test_gpu_attention8 import check
from token_cases import U16, U32

pytestmark = pytest.mark.gpu

# of the largest score of a tile, before the cap
PARTS = [1.0, 0.8, 0.55, 0.3, 0.1, -0.3, -0.6, -1.0]


def cancelling(codes, n, D, cap, reach):
    """A key head for each of PARTS, with one query head.  In each 64 places: 32 keys whose score before the cap is the part of `reach`, 31 of score 0, and one of
    score -reach (for negative parts reach) whose value is 0, so that every tile's largest score is `reach`.
    The values of the first two kinds are such that their weighted sum is nearly 0: what is left shows the scores' errors."""
    heads, places = len(PARTS), 640
    q = torch.zeros(1, n, heads, D, device="cuda")
    q[..., 0] = 2.0  # with a scale of 1/2 a score is its key's scale
    cache = pdx.new_cache(1, places, heads, D, codes)
    place = torch.arange(places, device="cuda")
    kind = torch.where(place % 64 == 63, 2, place % 2)  # 0: the part, 1: score 0, 2: the largest
    raw = torch.zeros(1, 2, heads, places, D, device="cuda")
    raw[:, 0, :, :, 0] = (kind != 1).float()
    raw[:, 1] = (kind != 2).float()[:, None]
    cache[0].copy_(raw.to(CODES[codes]))
    capped = (lambda s: cap * math.tanh(s / cap)) if cap else (lambda s: s)
    for h, part in enumerate(PARTS):
        s = part * reach if part > 0 else -min(-part * reach, 84.0 - capped(reach))  # (the smallest weights stay in fp32's range)
        s = float(torch.tensor(s))  # (as fp32 has it)
        cache[1][0, 0, h] = torch.where(kind == 0, s, -math.copysign(reach, part))
        s = capped(s)
        # values around 1 as the weights ask for; lifted where the third kind takes the weight
        lift = math.exp(min(capped(reach), 40.0)) if part < 0 else 1.0
        cache[1][0, 1, h] = torch.where(kind == 0, lift * math.exp(-s / 2) / 32, -lift * math.exp(s / 2) / 31)
    cache[2].zero_()
    return q.to(torch.bfloat16), cache, 0.5


def hold(codes, n, D, cap, reach, probability):
    """What cancelling values leave is within what scores and probabilities may be off by: probabilities times values' scales relative to themselves, and the
    header's 2^-20 of the cap (of the score above caps of 64)."""
    q, cache, scale = cancelling(codes, n, D, cap, reach)
    q_sites = torch.zeros(n, 4, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    pdx.attention8(q, cache, out, q_sites, scale=scale, cap=cap)
    torch.cuda.synchronize()
    want, moved, _ = tc.attention64(q, *mc.by_token(cache), q_sites[None], cache[2], scale, cap, None, False, -(1 << 31))
    # Scores: of the first kind alone, which is half of `moved`, as those of the second are 0.  The bound of the cap, and 8 roundings (key's scale, factor, product,
    # coefficients, sum with the reference).  The exponential's argument, up to 2^7 log2 units, is rounded, the exponential 2 u; then the sum over 640 keys.
    most = min(cap, reach) if cap else reach
    score = 2.0 ** -20 * (0.0 if not cap else cap if cap <= 64 else most) + 8 * U32 * most
    bound = U16 * want.abs() + moved * 1.01 * (probability + score / 2 + (130 + 640) * U32) + 1e-38
    off = (out.double() - want).abs()
    assert torch.all(off <= bound), (off / bound).amax((0, 1, 3))


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("largest", [0.3, 0.35, 0.45, 0.61, 0.7, 0.86, 1.0, 1.8])
@pytest.mark.parametrize("cap", [1.0, 20.0, 64.0])
def test_caps_up_to_64(codes, D, largest, cap):
    """Every tier of the polynomials.  Few rows keep probabilities times values' scales to 16 bits (2^-16), others to bf16."""
    hold(codes, 1, D, cap, largest * cap, 2.0 ** -16)
    hold(codes, 70, D, cap, largest * cap, U16)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("cap,largest", [(80.0, 0.3), (80.0, 0.7), (80.0, 1.5), (300.0, 0.2), (1e4, 0.004)])
def test_caps_above_64(codes, D, cap, largest):
    hold(codes, 1, D, cap, largest * cap, 2.0 ** -16)
    hold(codes, 70, D, cap, largest * cap, U16)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_without_a_cap(codes, D):
    for reach in (0.5, 20.0, 80.0):
        hold(codes, 1, D, 0.0, reach, 2.0 ** -16)
        hold(codes, 70, D, 0.0, reach, U16)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [32, 48, 64, 128])
@pytest.mark.parametrize("n", [65, 130])
def test_many_rows_keep_as_many_bits_as_few(codes, D, n):
    """16 bits of a probability times its value's scale, whatever the number of rows."""
    for cap, reach in ((0.0, 0.3), (0.0, 7.0), (20.0, 5.0), (20.0, 15.0), (80.0, 100.0)):
        hold(codes, n, D, cap, reach, 2.0 ** -16)


def ring(codes, g, d, kept, last, H, Hk, D):
    """A full ring of `kept` rounds up to round `last`, and its last round's sites."""
    grid = (d + 1) ** 2
    rounds = [pdx.volume_sites(d, 1, first_round=t) for t in range(last - kept + 1, last + 1)]
    sites = torch.cat(rounds)[None]
    turn = grid * ((last + 1) % kept)  # the place of the next round
    sites = torch.roll(sites, turn, 1)
    return mc.filled_cache(g, 1, kept * grid, Hk, D, codes, sites), rounds[-1][None]


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("last", [199, 256, 300, 355, 511, 1 << 20, 128, -1, 3])
@pytest.mark.parametrize("n", [1, 36])
def test_a_ring_at_any_round(codes, last, n):
    """200 rounds of d = 5, wherever the stream stands: inside one block of 256 rounds, across the border, behind it, below round 0."""
    g = tc.gen(last + n)
    cache, sites = ring(codes, g, 5, 200, last, 4, 2, 64)
    q = (3.0 * tc.normal(g, 1, n, 4, 64)).to(torch.bfloat16)
    slopes = torch.tensor([0.5, 0.1, 0.01, -0.05], device="cuda")
    check(q, cache, sites[:, :n], cap=30.0, slopes=slopes, causal=True)
    check(q, cache, sites[:, :n], slopes=slopes, causal=True)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
def test_a_ring_of_a_thousand_rounds(codes):
    g = tc.gen(51)
    cache, sites = ring(codes, g, 5, 1000, 5123, 4, 2, 32)
    slopes = torch.tensor([0.5, 0.1, 0.001, 0.0], device="cuda")
    for n in (1, 36):
        q = (3.0 * tc.normal(g, 1, n, 4, 32)).to(torch.bfloat16)
        check(q, cache, sites[:, :n], cap=30.0, slopes=slopes, causal=True)


def test_rows_of_rounds_on_both_sides_of_a_border():
    """Queries of several rounds, 254 to 258, as a call with a few rounds at once has them."""
    g = tc.gen(52)
    cache, _ = ring("e4m3", g, 5, 40, 260, 4, 2, 64)
    q_sites = torch.cat([pdx.volume_sites(5, 1, first_round=t) for t in range(254, 259)])[None]
    for m in (8, 180):
        q = (3.0 * tc.normal(g, 1, m, 4, 64)).to(torch.bfloat16)
        at = torch.arange(m, device="cuda") * 180 // m
        check(q, cache, q_sites[:, at].contiguous(), cap=30.0, slopes=torch.tensor([0.5, 0.1, 0.01, -0.05], device="cuda"), causal=True)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("n", [1, 70])
def test_scores_of_zero_under_the_smallest_caps(codes, n):
    """Keys up to 3e38 with queries of zeros: the key's scale over the cap leaves fp32's range, the scores are 0, and every value counts the same."""
    g = tc.gen(53)
    cache = mc.filled_cache(g, 1, 200, 1, 64, codes, torch.zeros(1, 200, 4, dtype=torch.int32, device="cuda"))
    cache[1][:, 0] = 3e38 / mc.QMAX[CODES[codes]]
    q_sites = torch.zeros(1, n, 4, dtype=torch.int32, device="cuda")
    q = torch.zeros(1, n, 2, 64, dtype=torch.bfloat16, device="cuda")
    v = mc.by_token(cache)[1][0].mean(0)
    for cap, scale in ((1e-5, 0.125), (0.0, 1e6)):
        out = torch.empty_like(q)
        pdx.attention8(q, cache, out, q_sites, cap=cap, scale=scale)
        torch.cuda.synchronize()
        moved = mc.by_token(cache)[1][0].abs().mean(0)
        assert torch.all((out.double() - v).abs() <= U16 * v.abs() + (U16 + 260 * U32) * 1.01 * moved)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("n", [1, 70])
def test_scores_under_the_largest_caps(codes, n):
    """Caps that no score comes near change nothing, whatever the keys' scales."""
    g = tc.gen(54)
    cache = mc.filled_cache(g, 1, 300, 2, 64, codes, torch.zeros(1, 300, 4, dtype=torch.int32, device="cuda"))
    cache[1][:, 0] *= 1e-5
    q = (2e5 * tc.normal(g, 1, n, 2, 64)).to(torch.bfloat16)
    q_sites = torch.zeros(1, n, 4, dtype=torch.int32, device="cuda")
    for cap in (1e30, 1e38, 3.4e38):
        out = torch.empty_like(q)
        pdx.attention8(q, cache, out, q_sites, cap=cap)
        torch.cuda.synchronize()
        # (such a cap is its own limit: tanh u = u)
        want, moved, score = tc.attention64(q, *mc.by_token(cache), q_sites, cache[2], 0.125, 0.0, None, False, -(1 << 31))
        z = (q.double().abs().amax() * mc.by_token(cache)[0].abs().amax()) * 64 * 0.125
        bound = tc.attention_tolerance(want, moved, score + (2.0 ** -20 + 4 * U32) * float(z))
        assert torch.all((out.double() - want).abs() <= bound)
