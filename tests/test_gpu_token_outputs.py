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


@pytest.mark.parametrize("order", list(itertools.permutations(range(3))))
@pytest.mark.parametrize("B,n,H", [(2, 50, 4), (1, 1, 4), (2, 7, 1)])
@pytest.mark.parametrize("pad", [0, 2])
def test_attention_outputs(order, B, n, H, pad):
    """Batch, tokens and heads in any order, next to each other and in wider rows."""
    g = tc.gen(B + n + H)
    q, k, v = (tc.normal(g, B, n, H, 64).to(torch.bfloat16) for _ in range(3))
    shape = [(B, n, H)[a] + pad for a in order] + [64]
    back = [order.index(0), order.index(1), order.index(2), 3]
    whole = torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")
    out = whole.permute(back)[:B, :n, :H]
    want, moved, score = tc.attention64(q, k, v, None, None, 0.125, 0.0, None, False, 0)
    pdx.attention(q, k, v, out)
    torch.cuda.synchronize()
    assert torch.all((out.double() - want).abs() <= tc.attention_tolerance(want, moved, score))
    out.fill_(7.0)
    assert torch.all(whole == 7.0)


def test_attention_outputs_on_each_other_are_refused():
    q = torch.zeros(2, 4, 4, 64, dtype=torch.bfloat16, device="cuda")
    for out in (q[:1].expand(2, 4, 4, 64), q[:, :1].expand(2, 4, 4, 64), q[:, :, :1].expand(2, 4, 4, 64)):
        with pytest.raises(pdx.PredecoderError) as e:
            pdx.attention(torch.zeros_like(q), q.clone(), q.clone(), out)
        assert e.value.status == pdx.PD_ERR_INVALID_ARG
