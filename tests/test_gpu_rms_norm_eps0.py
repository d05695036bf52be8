"""GPU: the root-mean-square norm where nothing is added below the root."""
import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu

WIDTHS = [5, 64, 96, 512, 1000, 2048, 4100, 8200]


def run(x, codes, gain=None, residual=None, eps=0.0):
    R, C = x.shape
    out = torch.full((R, C), 7.0, dtype=x.dtype, device="cuda")
    c = torch.full((R, C), 3, dtype=torch.int8, device="cuda").view(codes)
    sc = torch.full((R,), 7.0, device="cuda")
    pdx.rms_norm(x, gain, eps=eps, residual=residual, out=out, codes=c, scales=sc)
    torch.cuda.synchronize()
    return out, c, sc


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("codes", [torch.int8, torch.float8_e4m3fn])
def test_rows_of_zeros(width, dtype, codes):
    """A row of zeros has scale 0, codes 0 and output 0; also one whose gain is 0."""
    g = tc.gen(width)
    x = tc.normal(g, 7, width).to(tc.DTYPES[dtype])
    x[2] = x[5] = 0.0
    out, c, sc = run(x, codes)
    for n in (2, 5):
        assert sc[n] == 0 and torch.all(c[n].float() == 0) and torch.all(out[n] == 0)
    rest = [0, 1, 3, 4, 6]
    y = x[rest].double() / x[rest].double().square().mean(1, keepdim=True).sqrt()
    tc.check_codes(c[rest], sc[rest], y)
    assert torch.all((out[rest].double() - y).abs() <= (tc.UNIT[x.dtype] + tc.NORM_REL) * y.abs())
    out, c, sc = run(x, codes, gain=torch.zeros(width, device="cuda"), residual=torch.ones_like(x))
    assert torch.all(sc == 0) and torch.all(c.float() == 0) and torch.all(out == 0)
    minus = run(torch.zeros_like(x), codes, residual=-x)  # zeros by their sum
    assert minus[2][2] == 0 and torch.all(minus[0][2] == 0)
