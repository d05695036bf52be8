"""GPU: attention up to a token's own round where rounds are counted back from the present."""
import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu

NO_ROUND = -(1 << 31)  # no round is below it


@pytest.mark.parametrize("first", [-9, -4, -1000, 0, 5])
@pytest.mark.parametrize("d,T,D", [(3, 9, 64), (5, 9, 32), (7, 9, 128)])
@pytest.mark.parametrize("prefix", [None, 0, 2])
def test_rounds_below_zero(first, d, T, D, prefix):
    """Without a prefix no token sees a later round, negative ones neither; a prefix is all rounds below it."""
    g = tc.gen(d)
    sites = pdx.volume_sites(d, T, first_round=first)
    n = sites.shape[0]
    q, k, v = (tc.normal(g, 1, n, 2, D).to(torch.bfloat16) for _ in range(3))
    slopes = torch.tensor([0.5, 0.125], device="cuda")
    out = torch.full_like(q, 9.0)
    pdx.attention(q, k, v, out, sites, sites, slopes=slopes, causal=True, **({} if prefix is None else dict(prefix=prefix)))
    torch.cuda.synchronize()
    want, moved, score = tc.attention64(q, k, v, sites, sites, D ** -0.5, 0.0, slopes, True, NO_ROUND if prefix is None else prefix)
    assert torch.all((out.double() - want).abs() <= tc.attention_tolerance(want, moved, score))
    if prefix is None:  # later rounds do not reach earlier ones, whatever they hold
        later = (d + 1) ** 2 * 4
        k[:, later:] = v[:, later:] = float("nan")
        again = torch.full_like(q, 9.0)
        pdx.attention(q, k, v, again, sites, sites, slopes=slopes, causal=True)
        torch.cuda.synchronize()
        assert torch.equal(again[:, :later], out[:, :later])


def test_no_prefix_is_taken_with_and_without_causal():
    q = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    sites = torch.zeros(4, 4, dtype=torch.int32, device="cuda")
    for causal in (False, True):
        pdx.attention(q, q, q, torch.empty_like(q), sites, sites, causal=causal, prefix=None)
        assert pdx.attention_workspace(q, q, q, torch.empty_like(q), sites, sites, causal=causal) == 0
    with pytest.raises(pdx.PredecoderError):
        pdx.attention(q, q, q, torch.empty_like(q), sites, sites, causal=True, prefix=NO_ROUND + 1)
