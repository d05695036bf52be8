"""GPU: linear attention with a decay, over rounds, against its definition in 64 bits."""
import math

import pytest
import torch

import memory_cases as mc
import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu


def inputs(g, B, n, H, Hk, D):
    x = tc.normal(g, B, n, H + 2 * Hk, D).to(torch.bfloat16)
    return x[:, :, :H], x[:, :, H:H + Hk], x[:, :, H + Hk:]


def check(q, k, v, slopes, per_round, lengths=None, state=None, scale=None, in_place=False):
    B, n, H, D = q.shape
    Hk = k.shape[2]
    whole = torch.full((B, n, H, D + 8), 7.0, device="cuda", dtype=torch.bfloat16)
    out = whole[..., :D]
    given = None if state is None else state.clone()
    state_out = state if in_place else torch.full((B, Hk, D, D), 5.0, device="cuda")
    pdx.linear_attention(q, k, v, out, slopes=slopes, per_round=per_round, lengths=lengths, state=state, state_out=state_out, scale=scale)
    torch.cuda.synchronize()
    scale = D ** -0.5 if scale is None else scale
    want, S, out_size, size, rounds = mc.linear64(q, k, v, slopes, per_round, lengths, given, scale)
    bound, state_bound = mc.linear_tolerances(want, out_size, size, rounds, per_round, D)
    assert torch.all(whole[..., D:] == 7.0)
    for b in range(B):
        m = n if lengths is None else min(max(int(lengths[b]), 0), n)
        assert torch.all(out[b, m:] == 7.0)
        off = (out[b, :m].double() - want[b, :m]).abs()
        assert torch.all(off <= bound[b, :m]), (b, float((off / bound[b, :m]).amax()))
    off = (state_out.double() - S).abs()
    assert torch.all(off <= state_bound), float((off / state_bound).amax())
    return out, state_out


def slopes_of(Hk):
    return torch.exp2(-8.0 * (torch.arange(Hk, device="cuda") + 1.0) / Hk)


@pytest.mark.parametrize("B,n,per_round,H,Hk,D", [
    (1, 1, 1, 1, 1, 8), (3, 1, 1, 4, 2, 64), (2, 1, 1, 8, 8, 128), (1, 2, 1, 2, 1, 16), (1, 36, 36, 4, 4, 32), (2, 17, 1, 2, 2, 40), (1, 200, 1, 3, 3, 64),
    (1, 193, 2, 2, 1, 48), (2, 131, 5, 4, 2, 64), (1, 90, 9, 2, 2, 128), (1, 160, 16, 6, 2, 96), (1, 95, 31, 2, 2, 64), (1, 96, 32, 2, 2, 128),
    (2, 99, 33, 4, 1, 64), (1, 180, 36, 4, 4, 32), (1, 64, 64, 2, 2, 64), (1, 130, 65, 2, 2, 128), (1, 300, 100, 8, 2, 72), (2, 588, 196, 4, 2, 64),
    (1, 1000, 324, 2, 1, 128), (1, 1029, 1, 1, 1, 128), (4, 3, 7, 2, 2, 24), (1, 5, 2147483647, 2, 2, 64), (1, 7000, 1, 2, 1, 64), (1, 9800, 196, 2, 1, 32)])
def test_rounds(B, n, per_round, H, Hk, D):
    g = tc.gen(n * 10 + D)
    q, k, v = inputs(g, B, n, H, Hk, D)
    check(q, k, v, slopes_of(Hk), per_round)
    check(q, k, v, slopes_of(Hk), per_round, state=4.0 * tc.normal(g, B, Hk, D, D), in_place=True)
    check(q, k, v, None, per_round, scale=-0.5)


@pytest.mark.parametrize("per_round,n", [(1, 150), (1, 3), (5, 150), (36, 150), (64, 200), (100, 350)])
@pytest.mark.parametrize("D", [32, 128])
def test_lengths(per_round, n, D):
    """Entries of their own lengths (none, one, past the end); what lies behind them is neither read nor written."""
    g = tc.gen(n + D)
    lengths = torch.tensor([0, 1, n, n + 50, -3, n - 1, (n + 1) // 2], device="cuda", dtype=torch.int32)
    B = len(lengths)
    q, k, v = inputs(g, B, n, 4, 2, D)
    for b, m in enumerate(lengths.clamp(0, n).tolist()):
        for x in (q, k, v):
            x[b, m:] = math.nan
    state = tc.normal(g, B, 2, D, D)
    check(q, k, v, slopes_of(2), per_round, lengths)
    out, last = check(q, k, v, slopes_of(2), per_round, lengths, state)
    assert torch.equal(last[0], state[0]) and torch.equal(last[4], state[4])


@pytest.mark.parametrize("per_round,n", [(1, 130), (4, 130), (36, 144), (70, 280)])
def test_decays(per_round, n):
    """From none to all: a slope of 0 sums up, one of infinity leaves a round to itself."""
    g = tc.gen(per_round)
    q, k, v = inputs(g, 1, n, 5, 5, 64)
    slopes = torch.tensor([0.0, 1e-3, 3.0, 200.0, math.inf], device="cuda")
    check(q, k, v, slopes, per_round, state=tc.normal(g, 1, 5, 64, 64))


@pytest.mark.parametrize("per_round", [1, 3, 16, 40])
def test_later_rounds_do_not_reach_earlier_ones(per_round):
    """NaN and infinities in a round: results before it are as without; those from it on are not finite, and so is the state."""
    g = tc.gen(per_round + 50)
    n = 4 * per_round + 60
    q, k, v = inputs(g, 1, n, 2, 1, 64)
    clean, _ = check(q, k, v, slopes_of(1), per_round)
    at = (n // per_round // 2) * per_round
    for x, value in ((k, math.nan), (v, math.nan), (k, math.inf), (v, -math.inf)):
        kept = x[0, at, 0, 5].clone()
        x[0, at, 0, 5] = value
        out, state = torch.empty_like(clean), torch.empty(1, 1, 64, 64, device="cuda")
        pdx.linear_attention(q, k, v, out, slopes=slopes_of(1), per_round=per_round, state_out=state)
        torch.cuda.synchronize()
        x[0, at, 0, 5] = kept
        assert torch.equal(out[:, :at], clean[:, :at])
        hit = out[:, at:] if x is k else out[:, at:, :, 5]
        assert not torch.isfinite(hit).any()
        if x is v:  # the other columns stay
            rest = torch.cat([out[..., :5], out[..., 6:]], -1)
            assert torch.equal(rest, torch.cat([clean[..., :5], clean[..., 6:]], -1))
            assert torch.isfinite(state[..., :5]).all() and torch.isfinite(state[..., 6:]).all()
        hit = state[:, :, 5] if x is k else state[..., 5]
        assert not torch.isfinite(hit).any()


@pytest.mark.parametrize("per_round,parts", [(1, [1, 1, 1, 60, 3, 64, 70]), (4, [4, 4, 64, 128]), (36, [36, 36, 72]), (100, [100, 200])])
def test_piece_by_piece(per_round, parts):
    """A stream taken in pieces gives what it gives at once."""
    g = tc.gen(9)
    n = sum(parts)
    q, k, v = inputs(g, 2, n, 4, 2, 64)
    slopes, state = slopes_of(2), torch.zeros(2, 2, 64, 64, device="cuda")
    at, pieces = 0, []
    for m in parts:
        o = torch.empty(2, m, 4, 64, device="cuda", dtype=torch.bfloat16)
        pdx.linear_attention(q[:, at:at + m], k[:, at:at + m], v[:, at:at + m], o, slopes=slopes, per_round=per_round, state=state, state_out=state)
        pieces.append(o)
        at += m
    torch.cuda.synchronize()
    want, S, out_size, size, rounds = mc.linear64(q, k, v, slopes, per_round, None, None, 0.125)
    bound, state_bound = mc.linear_tolerances(want, out_size, size, rounds, per_round, 64)
    assert torch.all((torch.cat(pieces, 1).double() - want).abs() <= bound)
    assert torch.all((state.double() - S).abs() <= state_bound)


def test_streams_and_workspaces():
    g = tc.gen(10)
    q, k, v = inputs(g, 2, 5000, 4, 2, 64)
    slopes = slopes_of(2)
    a, b, c = (torch.empty(q.shape, dtype=q.dtype, device="cuda") for _ in range(3))
    pdx.linear_attention(q, k, v, a, slopes, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pdx.linear_attention(q, k, v, b, slopes, 4, stream=s)
    w = torch.empty(pdx.linear_attention_workspace(q, k, v, c, slopes, 4) + 16, dtype=torch.uint8, device="cuda")
    pdx.linear_attention(q, k, v, c, slopes, 4, workspace=w, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


def test_nothing_to_do():
    state = torch.randn(2, 2, 64, 64, device="cuda")
    out = torch.empty_like(state)
    e = torch.empty(2, 0, 2, 64, device="cuda", dtype=torch.bfloat16)
    pdx.linear_attention(e, e, e, e, per_round=3, state=state, state_out=out)
    torch.cuda.synchronize()
    assert torch.equal(state, out)
    pdx.linear_attention(e, e, e, e, state_out=out)
    torch.cuda.synchronize()
    assert torch.all(out == 0)


def test_refusals():
    q = torch.zeros(2, 6, 4, 64, device="cuda", dtype=torch.bfloat16)
    k = q[:, :, :2].contiguous()
    good = dict(q=q, k=k, v=k, out=torch.empty_like(q))
    for bad in (dict(q=q.float()), dict(k=k[:, :5]), dict(v=k[:1]), dict(out=q[:1]), dict(slopes=torch.zeros(4, device="cuda")),
                dict(lengths=torch.zeros(2, device="cuda")), dict(lengths=torch.zeros(3, device="cuda", dtype=torch.int32)),
                dict(state=torch.zeros(2, 2, 64, 32, device="cuda")), dict(state_out=torch.zeros(2, 2, 64, 64)), dict(k=k.clone().requires_grad_()),
                dict(state=torch.zeros(2, 2, 64, 64, device="cuda", dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            pdx.linear_attention(**(good | bad))
    for bad in (dict(per_round=0), dict(scale=math.inf), dict(out=q), dict(k=torch.cat([k, k[:, :, :1]], 2), v=torch.cat([k, k[:, :, :1]], 2))):
        with pytest.raises(pdx.PredecoderError) as e:
            pdx.linear_attention(**(good | bad))
        assert e.value.status == pdx.PD_ERR_INVALID_ARG
    q = torch.zeros(1, 2, 1, 136, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(pdx.PredecoderError) as e:
        pdx.linear_attention(q, q.clone(), q.clone(), torch.empty_like(q))
    assert e.value.status == pdx.PD_ERR_UNSUPPORTED
