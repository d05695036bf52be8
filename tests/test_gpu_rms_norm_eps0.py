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


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("codes", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("eps", [0.0, 1e-42, 1e-35, 1e-25])
def test_rows_of_tiny_values(width, dtype, codes, eps):
    """Rows whose squares leave fp32's range, down to its smallest numbers, next to usual ones."""
    g = tc.gen(width + 1)
    sizes = torch.tensor([0.0, -20.0, -44.0, -46.0, -60.0, -64.0, -75.0, -100.0, -120.0, -125.0, 10.0], dtype=torch.float64)
    x = (tc.normal(g, len(sizes), width).double() * torch.exp2(sizes).cuda()[:, None]).to(tc.DTYPES[dtype])
    gain = 1.0 + 0.3 * tc.normal(g, width)
    out, c, sc = run(x, codes, gain=gain, eps=eps)
    # (fp32 holds an eps below its normal range in few bits)
    e = torch.tensor(eps, dtype=torch.float32).double().item()
    y = x.double() / (x.double().square().mean(1, keepdim=True) + e).sqrt() * gain.double()
    assert torch.all((out.double() - y).abs() <= (tc.UNIT[x.dtype] + tc.NORM_REL) * y.abs() + 1e-38)
    big = y.abs().amax(1) > 1e-30  # (scales in the normal range)
    tc.check_codes(c[big], sc[big], y[big])


def test_one_tiny_value_in_a_wide_row():
    x = torch.zeros(3, 32768, device="cuda")
    x[0, 7], x[1, 32767], x[2, 0] = 1e-45, -1e-30, 1e-19
    out, c, sc = run(x, torch.int8)
    most = 32768 ** 0.5
    for n, at, sign in ((0, 7, 1), (1, 32767, -1), (2, 0, 1)):
        assert abs(float(out[n, at]) - sign * most) <= tc.NORM_REL * most + tc.U32 * most
        assert float(c[n, at]) == sign * 127 and int((c[n] != 0).sum()) == 1 and int((out[n] != 0).sum()) == 1
