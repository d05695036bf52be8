"""GPU: rotary positions over three axes against their definition in 64 bits."""
import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu


def places(g, n, most):
    t = torch.randint(0, most, (n, 4), generator=g, device="cuda", dtype=torch.int32)
    t[:, 1:3] %= 64
    t[::3, 1] *= -1
    return t


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,sections", [(1, 1, 2, (1, 0, 0)), (1, 3, 32, (8, 4, 4)), (36, 6, 64, (16, 8, 8)), (257, 5, 48, (12, 6, 6)),
                                                       (50, 2, 128, (20, 10, 10)), (13, 7, 30, (5, 5, 5)), (9, 16, 256, (64, 32, 32)),
                                                       (700, 10, 64, (0, 16, 16)), (5, 1, 96, (0, 0, 0))])
def test_turns(dtype, interleaved, inverse, tokens, heads, dim, sections):
    g = tc.gen(tokens * 100 + dim)
    dt = tc.DTYPES[dtype]
    x = tc.normal(g, tokens, heads, dim).to(dt)
    sites = places(g, tokens, 1000)
    out = torch.full_like(x, 9.0)
    pdx.rope(x, sites, out, sections, base=100.0, interleaved=interleaved, inverse=inverse)
    torch.cuda.synchronize()
    want = tc.rope64(x, sites, sections, 100.0, interleaved, inverse)
    assert torch.all((out.double() - want).abs() <= tc.rope_tolerance(x, want, interleaved))
    rest = dim // 2 - sum(sections)
    if rest:  # the pairs past the sections are copied
        cut = 2 * sum(sections) if interleaved else sum(sections)
        same = (out[..., cut:], x[..., cut:]) if interleaved else (out[..., cut:dim // 2], x[..., cut:dim // 2])
        assert torch.equal(*same)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_late_rounds(dtype):
    """Angles of rounds in the millions are as exact as those of the first."""
    g = tc.gen(3)
    x = tc.normal(g, 64, 2, 64).to(tc.DTYPES[dtype])
    sites = places(g, 64, 1 << 22)
    sites[0, 0] = (1 << 23) - 1
    out = torch.empty_like(x)
    pdx.rope(x, sites, out, (16, 8, 8))
    torch.cuda.synchronize()
    want = tc.rope64(x, sites, (16, 8, 8), 10000.0, False, False)
    # base^(-k/n) times 2^23 has an error of 2^23 2^-53 in the 64-bit reference: nothing here
    assert torch.all((out.double() - want).abs() <= tc.rope_tolerance(x, want, False))


@pytest.mark.parametrize("pad,shift", [(2, 0), (0, 1), (1, 3)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_in_wider_rows(dtype, pad, shift, interleaved):
    g = tc.gen(pad * 10 + shift)
    dt = tc.DTYPES[dtype]
    n, H, D = 77, 6, 64
    whole = tc.normal(g, n * (H + pad) * D + shift).to(dt)
    x = whole[shift:].view(n, H + pad, D)[:, :H]
    before, kept = x.clone(), whole.clone()
    sites = places(g, n, 50)
    pdx.rope(x, sites, x, (16, 8, 8), interleaved=interleaved)
    torch.cuda.synchronize()
    want = tc.rope64(before, sites, (16, 8, 8), 10000.0, interleaved, False)
    assert torch.all((x.double() - want).abs() <= tc.rope_tolerance(before, want, interleaved))
    whole[shift:].view(n, H + pad, D)[:, :H] = before
    assert torch.equal(whole, kept)  # nothing outside was written


def test_back_and_forth_and_gradient():
    """The inverse undoes the turn, and is its gradient: <R x, y> = <x, R^-1 y>; differences agree."""
    g = tc.gen(11)
    x, y = (tc.normal(g, 40, 3, 64) for _ in range(2))
    sites = places(g, 40, 300)
    a, b, c = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    pdx.rope(x, sites, a, (16, 8, 8))
    pdx.rope(a, sites, b, (16, 8, 8), inverse=True)
    pdx.rope(y, sites, c, (16, 8, 8), inverse=True)
    torch.cuda.synchronize()
    pair = x.abs()[..., :32] + x.abs()[..., 32:]
    assert torch.all((b - x).abs() <= 4 * (4 * 3.15 + 8) * tc.U32 * pair.repeat(1, 1, 2))
    n = x.numel()
    left, right = (a.double() * y.double()).sum(), (x.double() * c.double()).sum()
    size = float((a.double().norm() * y.double().norm()))
    assert abs(float(left - right)) <= 2 * (4 * 3.15 + 8) * tc.U32 * size * 2
    # the derivative of <R x, y> along e by a central difference of the kernel itself (R is linear: no remainder)
    e = tc.normal(g, 40, 3, 64)
    up, down = torch.empty_like(x), torch.empty_like(x)
    pdx.rope(x + e, sites, up, (16, 8, 8))
    pdx.rope(x - e, sites, down, (16, 8, 8))
    torch.cuda.synchronize()
    slope = ((up.double() - down.double()) * y.double()).sum() / 2
    assert abs(float(slope - (c.double() * e.double()).sum())) <= 8 * (4 * 3.15 + 8) * tc.U32 * float(y.double().norm()) * float(
        x.double().norm() + e.double().norm()) and n > 0


def test_no_tokens_and_other_stream():
    e = torch.empty(0, 2, 32, device="cuda")
    pdx.rope(e, torch.empty(0, 4, dtype=torch.int32, device="cuda"), e, (8, 4, 4))
    g = tc.gen(2)
    x, sites = tc.normal(g, 3000, 4, 64), places(g, 3000, 99)
    out, again = torch.empty_like(x), torch.empty_like(x)
    pdx.rope(x, sites, out, (16, 8, 8))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pdx.rope(x, sites, again, (16, 8, 8), stream=s)
    torch.cuda.synchronize()
    assert torch.equal(out, again)


def test_refusals():
    x = torch.zeros(4, 2, 32, device="cuda")
    sites = torch.zeros(4, 4, dtype=torch.int32, device="cuda")
    for bad in (dict(sites=sites[:3]), dict(sites=sites.long()), dict(sites=sites[:, :3]), dict(sites=sites.cpu()),
                dict(out=x.half()), dict(out=x[:3]), dict(out=x.cpu()), dict(out=torch.zeros(4, 32, 2, device="cuda").transpose(1, 2))):
        a = dict(x=x, sites=sites, out=torch.empty_like(x), sections=(8, 4, 4)) | bad
        with pytest.raises(ValueError):
            pdx.rope(**a)
    for bad in (dict(sections=(9, 4, 4)), dict(sections=(-1, 4, 4)), dict(base=0.0), dict(base=float("nan"))):
        with pytest.raises(pdx.PredecoderError) as e:
            pdx.rope(x, sites, torch.empty_like(x), **(dict(sections=(8, 4, 4)) | bad))
        assert e.value.status == pdx.PD_ERR_INVALID_ARG
    y = torch.zeros(4, 1, 258, device="cuda")
    with pytest.raises(pdx.PredecoderError) as e:
        pdx.rope(y, sites, torch.empty_like(y), (8, 4, 4))
    assert e.value.status == pdx.PD_ERR_UNSUPPORTED
    y = torch.zeros(4, 2, 31, device="cuda")
    with pytest.raises(pdx.PredecoderError) as e:
        pdx.rope(y, sites, torch.empty_like(y), (1, 1, 1))
    assert e.value.status == pdx.PD_ERR_INVALID_ARG
