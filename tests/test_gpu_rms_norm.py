"""GPU: the root-mean-square norm against its definition in 64 bits."""
import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu


def rows_of(g, rows, width, dtype, pad=0, shift=0):
    """[rows][width] inside rows of `pad` more values, `shift` values past an aligned address."""
    t = tc.normal(g, rows * (width + pad) + shift) * 2.0
    return t.to(dtype)[shift:].view(rows, width + pad)[:, :width]


def run(x, gain, residual, codes_dtype, want_out=True):
    R, C = x.shape
    s = torch.full_like(x, 7.0, memory_format=torch.contiguous_format) if residual is not None else None
    out = torch.full((R, C), 7.0, dtype=x.dtype, device="cuda") if want_out else None
    codes = scales = None
    if codes_dtype is not None:
        codes = torch.full((R, C), 3, dtype=torch.int8, device="cuda").view(codes_dtype)
        scales = torch.full((R,), 7.0, device="cuda")
    pdx.rms_norm(x, gain, eps=tc.EPS, residual=residual, sum_out=s, out=out, codes=codes, scales=scales)
    torch.cuda.synchronize()
    return s, out, codes, scales


# widths around each lane count and granule, odd ones, the widest; one row, rows that leave a workgroup's last places empty
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 5), (1, 8), (33, 64), (7, 72), (5, 128), (180, 129), (65, 256), (9, 333), (4, 512),
                                        (6, 520), (3, 1024), (2, 1111), (5, 2048), (3, 2056), (2, 4097), (2, 8192), (1, 8200),
                                        (2, 32768)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("codes", [None, torch.int8, torch.float8_e4m3fn])
def test_rows(rows, width, dtype, codes):
    g = tc.gen(rows * 40009 + width)
    dt = tc.DTYPES[dtype]
    x, r = rows_of(g, rows, width, dt), rows_of(g, rows, width, dt)
    gain = 1.0 + 0.3 * tc.normal(g, width)
    s, out, c, sc = run(x, gain, r, codes)
    s64, y = tc.norm64(x, r, gain)
    u = tc.UNIT[dt]
    assert torch.all((s.double() - s64).abs() <= (u + tc.U32) * s64.abs())
    assert torch.all((out.double() - y).abs() <= (u + tc.NORM_REL) * y.abs() + tc.NORM_REL * 1e-3)
    if codes is not None:
        tc.check_codes(c, sc, y)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (16, 8)])
@pytest.mark.parametrize("residual", [False, True])
def test_strides_and_alignment(dtype, pad, shift, residual):
    g = tc.gen(pad * 17 + shift)
    dt = tc.DTYPES[dtype]
    x = rows_of(g, 50, 264, dt, pad, shift)
    r = rows_of(g, 50, 264, dt, 8) if residual else None
    s, out, c, sc = run(x, None, r, torch.int8)
    s64, y = tc.norm64(x, r, None)
    assert torch.all((out.double() - y).abs() <= (tc.UNIT[dt] + tc.NORM_REL) * y.abs())
    tc.check_codes(c, sc, y)


def test_many_rows_past_the_grid():
    """More rows than the largest launch has places for."""
    rows = (1 << 21) * 32 + 77
    x = torch.zeros(rows, 8, dtype=torch.bfloat16, device="cuda")
    x[:, 0] = (torch.arange(rows, device="cuda") % 251 + 1).to(torch.bfloat16)
    out = torch.zeros_like(x)
    pdx.rms_norm(x, eps=0.0, out=out)
    torch.cuda.synchronize()
    assert torch.all(out[:, 0] == torch.tensor(8.0 ** 0.5, dtype=torch.bfloat16, device="cuda")) and torch.all(out[:, 1:] == 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_place(dtype):
    g = tc.gen(5)
    dt = tc.DTYPES[dtype]
    x, r = rows_of(g, 300, 512, dt), rows_of(g, 300, 512, dt)
    s64, y = tc.norm64(x, r, None)
    pdx.rms_norm(x, residual=r, sum_out=r, out=x, eps=tc.EPS)
    torch.cuda.synchronize()
    u = tc.UNIT[dt]
    assert torch.all((r.double() - s64).abs() <= (u + tc.U32) * s64.abs())
    assert torch.all((x.double() - y).abs() <= (u + tc.NORM_REL) * y.abs() + 1e-9)


@pytest.mark.parametrize("codes", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("width", [96, 100, 4096])
def test_rows_of_zeros_tiny_huge_and_not_finite(codes, width):
    x = torch.ones(8, width, device="cuda")
    x[0] = 0.0
    x[1] = 1e-38
    x[2, 1:] = 1e-39  # subnormal but for one value
    x[3] = 1e25       # the sum of squares overflows
    x[4, 3] = float("inf")
    x[5, 3] = float("nan")
    x[6, 5] = 100.0
    s, out, c, sc = run(x, None, None, codes)
    v = c.double()
    q = 127.0 if codes == torch.int8 else 448.0
    assert sc[0] == 0 and torch.all(v[0] == 0) and torch.all(out[0] == 0)
    assert torch.all(v[1] == q)
    assert v[2, 0] == q and torch.all(v[2, 1:] == 0)
    for n in (3, 4, 5):
        assert torch.isnan(sc[n]) and torch.all(v[n] == 0)
    assert v[6, 5] == q and torch.isfinite(sc[[1, 2, 6, 7]]).all()
    assert torch.isnan(out[5]).all()
    tc.check_codes(c[6:], sc[6:], tc.norm64(x[6:], None, None)[1])


def test_a_gain_that_is_not_finite_marks_the_row():
    x = torch.ones(2, 64, device="cuda")
    gain = torch.ones(64, device="cuda")
    gain[5] = float("nan")
    _, out, c, sc = run(x, gain, None, torch.int8)
    assert torch.isnan(sc).all() and torch.all(c == 0)
    assert torch.isnan(out[:, 5]).all() and torch.isfinite(out[:, :5]).all()


def test_other_stream_and_no_rows():
    g = tc.gen(9)
    x = rows_of(g, 4000, 512, torch.bfloat16)
    out, again = torch.empty_like(x), torch.empty_like(x)
    pdx.rms_norm(x, out=out)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pdx.rms_norm(x, out=again, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    e = torch.empty(0, 64, device="cuda")
    pdx.rms_norm(e, out=e.clone())
    torch.cuda.synchronize()


def test_refusals():
    x = torch.zeros(4, 64, device="cuda")
    out, codes, sc = torch.empty_like(x), torch.empty(4, 64, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    for bad in (dict(), dict(out=out.half()), dict(out=out[:3]), dict(out=out.cpu()), dict(codes=codes), dict(scales=sc, out=out),
                dict(out=out, gain=torch.zeros(63, device="cuda")), dict(out=out, residual=x.to(torch.bfloat16)),
                dict(codes=codes.view(torch.uint8), scales=sc), dict(codes=codes, scales=sc[:2])):
        with pytest.raises(ValueError):
            pdx.rms_norm(x, **bad)
    with pytest.raises(ValueError):
        pdx.rms_norm(x.t(), out=torch.empty(64, 4, device="cuda"))
    with pytest.raises(pdx.PredecoderError) as e:
        pdx.rms_norm(torch.zeros(1, 32769, device="cuda"), out=torch.zeros(1, 32769, device="cuda"))
    assert e.value.status == pdx.PD_ERR_UNSUPPORTED
    for eps in (-1.0, float("nan")):
        with pytest.raises(pdx.PredecoderError) as e:
            pdx.rms_norm(x, out=out, eps=eps)
        assert e.value.status == pdx.PD_ERR_INVALID_ARG
    with pytest.raises(pdx.PredecoderError):  # rows of the output on top of each other
        pdx.rms_norm(x, out=torch.zeros(64, device="cuda").expand(4, 64))


@pytest.mark.parametrize("width", [64, 512, 1024])
def test_results_larger_than_the_caches(width):
    """Results that are stored past the caches are the same as those of the rows one part at a time."""
    rows = (129 << 20) // (2 * width)
    g = tc.gen(width)
    x, r = rows_of(g, rows, width, torch.bfloat16), rows_of(g, rows, width, torch.bfloat16)
    whole = run(x, None, r, torch.float8_e4m3fn)
    n = rows // 3
    for lo in (0, n, 2 * n):
        for a, b in zip(whole, run(x[lo:lo + n], None, r[lo:lo + n], torch.float8_e4m3fn)):
            assert torch.equal(a[lo:lo + n].view(torch.uint8), b.view(torch.uint8))
    s64, y = tc.norm64(x[-999:], r[-999:], None)
    assert torch.all((whole[0][-999:].double() - s64).abs() <= (tc.U16 + tc.U32) * s64.abs())
    assert torch.all((whole[1][-999:].double() - y).abs() <= (tc.U16 + tc.NORM_REL) * y.abs())
