"""GPU: the weights of attention add up to one, as the header says: their sum is that of the rounded probabilities."""
import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 5000), (40, 63), (300, 700), (130, 20000)])
@pytest.mark.parametrize("cap", [0.0, 30.0, 1e4])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_equal_values_come_out_as_they_are(nq, nk, cap, D):
    """sum p v / sum p of one v for all keys is v: the sums differ by fp32 roundings alone, far below half a bf16 step."""
    g = tc.gen(nq + nk)
    q, k = ((1.5 * tc.normal(g, 2, n, 2, D)).to(torch.bfloat16) for n in (nq, nk))
    v = tc.normal(g, 2, 1, 2, D).to(torch.bfloat16).expand(2, nk, 2, D).contiguous()
    out = torch.full_like(q, 9.0)
    pdx.attention(q, k, v, out, cap=cap)
    torch.cuda.synchronize()
    assert torch.equal(out, v[:, :1].expand(2, nq, 2, D))
