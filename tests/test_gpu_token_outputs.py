"""GPU: outputs of the token operators in every order of their axes, which the check of their strides lets through."""
import itertools

import pytest
import torch

import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("order", list(itertools.permutations(range(2))))
@pytest.mark.parametrize("tokens,heads", [(1, 1), (1, 3), (50, 1), (50, 3)])
@pytest.mark.parametrize("pad", [0, 2])
def test_rotary_outputs(order, tokens, heads, pad):
    """Tokens before heads and heads before tokens, next to each other and in wider rows, in place and not."""
    g = tc.gen(tokens + heads)
    x = tc.normal(g, tokens, heads, 32)
    sites = torch.randint(0, 9, (tokens, 4), generator=g, device="cuda", dtype=torch.int32)
    shape = [(tokens, heads)[k] + pad for k in order] + [32]
    back = [order.index(0), order.index(1), 2]
    whole = torch.full(shape, 7.0, device="cuda")
    out = whole.permute(back)[:tokens, :heads]
    want = tc.rope64(x, sites, (8, 4, 4), 10000.0, False, False)
    pdx.rope(x, sites, out, (8, 4, 4))
    torch.cuda.synchronize()
    assert torch.all((out.double() - want).abs() <= tc.rope_tolerance(x, want, False))
    out.copy_(x)
    pdx.rope(out, sites, out, (8, 4, 4))
    torch.cuda.synchronize()
    assert torch.all((out.double() - want).abs() <= tc.rope_tolerance(x, want, False))
    out.fill_(7.0)
    assert torch.all(whole == 7.0)


def test_rotary_outputs_on_each_other_are_refused():
    x = torch.zeros(5, 3, 32, device="cuda")
    sites = torch.zeros(5, 4, dtype=torch.int32, device="cuda")
    for out in (x[:1].expand(5, 3, 32), x[:, :1].expand(5, 3, 32), torch.zeros(300, device="cuda").as_strided((5, 3, 32), (40, 16, 1))):
        with pytest.raises(pdx.PredecoderError) as e:
            pdx.rope(torch.zeros_like(x), sites, out, (8, 4, 4))
        assert e.value.status == pdx.PD_ERR_INVALID_ARG
