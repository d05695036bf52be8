"""GPU: linear attention over rounds that are cut into segments (a state pass, a scan, a result pass), against its definition in 64 bits."""
import math

import pytest
import torch

import memory_cases as mc
import paper_2604_12841_amd as pdx
import token_cases as tc

pytestmark = pytest.mark.gpu

N, H, HK = 3000, 6, 3


def segment_tokens(B, per_round, D):
    """Tokens of a segment, as the library plans it; checked against the workspace that it asks for."""
    rounds = -(-N // per_round)
    tile_rounds = (64 if D <= 64 else 48) // per_round if per_round <= 32 else 1
    most = N // max(256, 4 * D)
    segments = max(1, min((2048 if D <= 32 else 512 if D <= 64 else 256) // (B * HK), most))
    each = -(-(-(-rounds // segments)) // tile_rounds) * tile_rounds
    q = torch.empty(B, N, H, D, device="cuda", dtype=torch.bfloat16)
    need = pdx.linear_attention_workspace(q, q[:, :, :HK], q[:, :, :HK], torch.empty_like(q), None, per_round)
    assert need == B * HK * -(-rounds // each) * D * D * 4 and rounds > 2 * each
    return each * per_round


def rounds64(q, k, v, slopes, per_round, lengths, state, scale):
    """The definition in 64 bits, all entries and heads of a round together: (out, state, the same sums of absolute values)."""
    B, n, H, D = q.shape
    Hk = k.shape[2]
    count = torch.full((B,), n, device="cuda") if lengths is None else lengths.clamp(0, n).long()
    there = torch.arange(n, device="cuda")[None] < count[:, None]
    q, k, v = (torch.where(there[..., None, None], x.double(), 0.0).transpose(1, 2).contiguous() for x in (q, k, v))
    fade = torch.ones(Hk, device="cuda", dtype=torch.float64) if slopes is None else torch.exp(-slopes.double())
    s = torch.zeros(B, Hk, D, D, device="cuda", dtype=torch.float64) if state is None else state.double()
    a = s.abs()
    out = torch.zeros(B, H, n, D, device="cuda", dtype=torch.float64)
    size = torch.zeros_like(out)
    for lo in range(0, n, per_round):
        hi = min(n, lo + per_round)
        on = (count > lo)[:, None, None, None]
        kk, vv = k[:, :, lo:hi].transpose(2, 3).contiguous(), v[:, :, lo:hi].contiguous()
        s = torch.where(on, s * fade[:, None, None] + kk @ vv, s)
        a = torch.where(on, a * fade[:, None, None] + kk.abs() @ vv.abs(), a)
        qq = q[:, :, lo:hi].reshape(B, Hk, -1, D)
        out[:, :, lo:hi] = (scale * (qq @ s)).view(B, H, hi - lo, D)
        size[:, :, lo:hi] = (abs(scale) * (qq.abs() @ a)).view(B, H, hi - lo, D)
    rounds = [-(-int(m) // per_round) for m in count]
    return out.transpose(1, 2), s, size.transpose(1, 2), a, rounds


def inputs(g, B, D):
    x = tc.normal(g, B, N, H + 2 * HK, D).to(torch.bfloat16)
    return x[:, :, :H], x[:, :, H:H + HK], x[:, :, H + HK:]


@pytest.mark.parametrize("per_round", [1, 5, 32, 33, 36, 196])
@pytest.mark.parametrize("D", [32, 40, 64, 128])
def test_entries_of_their_own_lengths(per_round, D):
    """No tokens, one, ends beside and at the segments' ends, inside rounds; with and without a state before; no decay, a slow one, nothing but a round."""
    g = tc.gen(per_round * 100 + D)
    seg = segment_tokens(8, per_round, D)
    lengths = torch.tensor([0, 1, seg - 1, seg, seg + 1, 2 * seg, N - 1, N + 7], device="cuda", dtype=torch.int32)
    B = len(lengths)
    q, k, v = inputs(g, B, D)
    for b, m in enumerate(lengths.clamp(0, N).tolist()):
        for x in (q, k, v):
            x[b, m:] = math.nan
    slopes = torch.tensor([0.0, 0.02, math.inf], device="cuda")
    for given in (None, 4.0 * tc.normal(g, B, HK, D, D)):
        out = torch.full((B, N, H, D), 7.0, device="cuda", dtype=torch.bfloat16)
        state = torch.full((B, HK, D, D), 5.0, device="cuda") if given is None else given.clone()
        pdx.linear_attention(q, k, v, out, slopes=slopes, per_round=per_round, lengths=lengths, state=None if given is None else state, state_out=state)
        torch.cuda.synchronize()
        want, S, out_size, size, rounds = rounds64(q, k, v, slopes, per_round, lengths, given, D ** -0.5)
        bound, state_bound = mc.linear_tolerances(want, out_size, size, rounds, per_round, D)
        for b, m in enumerate(lengths.clamp(0, N).tolist()):
            assert torch.all(out[b, m:] == 7.0)
            off = (out[b, :m].double() - want[b, :m]).abs()
            assert torch.all(off <= bound[b, :m]), (b, float((off / bound[b, :m]).amax()))
        off = (state.double() - S).abs()
        assert torch.all(off <= state_bound), float((off / state_bound).amax())
        assert torch.equal(state[0], torch.zeros_like(state[0]) if given is None else given[0])


@pytest.mark.parametrize("per_round", [1, 5, 36, 196])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_what_is_not_finite_reaches_later_segments_alone(per_round, D):
    g = tc.gen(per_round + D)
    seg = segment_tokens(1, per_round, D)
    q, k, v = inputs(g, 1, D)
    slopes = torch.tensor([0.0, 0.01, 0.3], device="cuda")

    def run():
        out, state = torch.empty(1, N, H, D, device="cuda", dtype=torch.bfloat16), torch.empty(1, HK, D, D, device="cuda")
        pdx.linear_attention(q, k, v, out, slopes=slopes, per_round=per_round, state_out=state)
        torch.cuda.synchronize()
        return out, state
    clean, last = run()
    at = (seg + seg // 2) // per_round * per_round  # in the middle of the second segment, of three at least
    for x, value in ((k, math.nan), (v, math.nan), (k, math.inf), (v, -math.inf)):
        kept = x[0, at, 1, 5].clone()
        x[0, at, 1, 5] = value
        out, state = run()
        x[0, at, 1, 5] = kept
        assert torch.equal(out[:, :at], clean[:, :at])
        others = [0, 1, 4, 5]  # query heads of the other key heads
        assert torch.equal(out[:, :, others], clean[:, :, others]) and torch.equal(state[:, [0, 2]], last[:, [0, 2]])
        hit = out[:, at:, 2:4] if x is k else out[:, at:, 2:4, 5]
        assert not torch.isfinite(hit).any()
        assert not torch.isfinite(state[:, 1, 5] if x is k else state[:, 1, :, 5]).any()
        if x is v:
            columns = [c for c in range(D) if c != 5]
            assert torch.equal(out[..., columns], clean[..., columns]) and torch.equal(state[..., columns], last[..., columns])


@pytest.mark.parametrize("n,per_round,D", [(1, 1, 8), (1, 1, 72), (3, 1, 8), (3, 40, 8), (3, 1, 72), (3, 40, 72)])
def test_many_entries(n, per_round, D):
    """131200 entries' heads: each as in a call of fewer."""
    B, Hk, part = 16400, 8, 4100
    g = tc.gen(n + D)
    x = tc.normal(g, B, n, 2 * Hk, D).to(torch.bfloat16)
    q, k = x[:, :, :Hk], x[:, :, Hk:]
    state = tc.normal(g, B, Hk, D, D) if D == 8 else None
    slopes = torch.linspace(0.0, 1.0, Hk, device="cuda")
    out, want = torch.empty(B, n, Hk, D, device="cuda", dtype=torch.bfloat16), torch.empty(B, n, Hk, D, device="cuda", dtype=torch.bfloat16)
    last, want_last = (None, None) if state is None else (torch.empty_like(state), torch.empty_like(state))
    pdx.linear_attention(q, k, k, out, slopes=slopes, per_round=per_round, state=state, state_out=last)
    for b in range(0, B, part):
        s = slice(b, b + part)
        pdx.linear_attention(q[s], k[s], k[s], want[s], slopes=slopes, per_round=per_round, state=None if state is None else state[s],
                             state_out=None if state is None else want_last[s])
    torch.cuda.synchronize()
    assert torch.equal(out, want) and (state is None or torch.equal(last, want_last))
