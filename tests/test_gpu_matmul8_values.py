"""GPU: the product of 8-bit codes where values are not finite or cancel."""
import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N", [(4, 96), (300, 3000), (2100, 2100), (4096, 4096)])  # every kernel
def test_marked_rows_stay_marked(act, kind, out, M, N):
    """A row that the norm marked (scale NaN, codes 0) is NaN behind every activation, and no other row is."""
    g = tc.gen(M)
    a, w = (torch.randint(-20, 21, (n, 64), generator=g, device="cuda").to(torch.float32).to(CODES[kind]) for n in (M, N))
    a[1] = 0
    sa, sw = torch.full((M,), 0.01, device="cuda"), torch.full((N,), 0.01, device="cuda")
    sa[1] = float("nan")
    b = tc.normal(g, N)
    b[5] = float("nan")
    o = torch.empty(M, N, dtype=tc.DTYPES[out], device="cuda")
    pdx.matmul8(a, sa, w, sw, o, bias=b, act=act)
    torch.cuda.synchronize()
    assert torch.isnan(o[1]).all() and torch.isnan(o[:, 5]).all()
    o[1] = o[:, 5] = 0.0
    assert torch.isfinite(o).all()


def cancelling(g, M, N, K, small):
    """E4M3 codes whose products cancel: a large pair of opposite signs among small values, in random places."""
    a, w = (small * torch.randint(1, 3, (n, K), generator=g, device="cuda").float() for n in (M, N))
    at = torch.argsort(torch.rand(M, K, generator=g, device="cuda"), 1)[:, :2]
    rows = torch.arange(M, device="cuda")
    a[rows, at[:, 0]], a[rows, at[:, 1]] = 448.0, -448.0
    w[:, at[: min(M, 8)].flatten()] = 448.0  # the places of the first rows' pairs
    return a.to(CODES["e4m3"]), w.to(CODES["e4m3"])


@pytest.mark.parametrize("M,N,K", [(8, 33, 64), (8, 512, 512), (200, 96, 1000), (2100, 2100, 128), (4096, 4096, 64)])  # every kernel
@pytest.mark.parametrize("small", [2.0 ** -9, 2.0 ** -3, 1.0, 4.0])
@pytest.mark.parametrize("bias", [False, True])
def test_e4m3_sums_that_cancel(M, N, K, small, bias):
    """To fp32 the sums are fp32's.  To bf16 each product loses less than 2^-13 of the largest of its eight neighbours, which
    the largest itself does not lose; more where sums cancel than the output's rounding."""
    g = tc.gen(M + N + K)
    a, w = cancelling(g, M, N, K, small)
    one = torch.ones(max(M, N), device="cuda")
    want, size = tc.matmul64(a, one[:M], w, one[:N], None, "none")
    b = None
    if bias:  # nearly what the first row's sum is without its sign
        b = -want[0].float() * (1 + 2.0 ** -10)
        want = want + b.double()
    # 7 2^-13 of every eight's largest |product|: at most the largest |a| times the largest |w| of the eight
    pad = (-K) % 8
    most = [torch.nn.functional.pad(t.float().abs(), (0, pad)).view(t.shape[0], -1, 8).amax(2).double() for t in (a, w)]
    eights = 7 * 2.0 ** -13 * (most[0] @ most[1].t().contiguous())
    extra = 0.0 if b is None else b.double().abs()
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.empty(M, N, dtype=dtype, device="cuda")
        pdx.matmul8(a, one[:M], w, one[:N], out, bias=b)
        torch.cuda.synchronize()
        part = K * tc.U32 * size + 4 * tc.U32 * (size + extra) + (eights if dtype == torch.bfloat16 else 0.0)
        assert torch.all((out.double() - want).abs() <= part + tc.UNIT[dtype] * (want.abs() + part))
