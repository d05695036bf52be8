"""Host-side checks of the token operators' outputs whose rows lie on each other: refused before any device call."""
import ctypes

import pytest

import paper_2604_12841_amd as pdx
from paper_2604_12841_amd import tokens

P = 4096  # an aligned address that no call may touch
BAD = pdx.PD_ERR_INVALID_ARG


def rope(**kw):
    a = dict(tokens=5, heads=3, head_dim=32, dtype=1, sections=(8, 4, 4), base=100.0, sites=P, x=2 * P, x_token_stride=96, x_head_stride=32, out=P,
             out_token_stride=96, out_head_stride=32) | kw
    a["sections"] = (ctypes.c_int32 * 3)(*a["sections"])
    return tokens._functions().predecoder_rope(None, tokens.RopeArgs(**a))


@pytest.mark.parametrize("kw", [dict(out_token_stride=0), dict(out_head_stride=0), dict(out_head_stride=31), dict(out_token_stride=95),
                                dict(out_token_stride=-95), dict(out_token_stride=32, out_head_stride=159), dict(out_token_stride=-(1 << 63), tokens=1 << 30, out_head_stride=0),
                                # x itself, under other strides
                                dict(out=2 * P, out_token_stride=128), dict(out=2 * P, out_token_stride=32, out_head_stride=160)])
def test_rotary_outputs_on_each_other(kw):
    assert rope(**kw) == BAD


def attention(**kw):
    a = dict(batch=2, heads=4, kv_heads=2, head_dim=64, n_q=4, n_k=9, scale=0.1)
    for n in ("q", "k", "v", "out"):
        a |= {n: P, n + "_batch_stride": 1024, n + "_token_stride": 256, n + "_head_stride": 64}
    return tokens._functions().predecoder_attention(None, tokens.AttentionArgs(**(a | kw)))


@pytest.mark.parametrize("kw", [dict(out_batch_stride=0), dict(out_token_stride=0), dict(out_head_stride=0), dict(out_head_stride=56),
                                dict(out_token_stride=248), dict(out_token_stride=-248), dict(out_batch_stride=1016),
                                dict(out_token_stride=64, out_head_stride=248), dict(out_batch_stride=256, out_token_stride=504)])
def test_attention_outputs_on_each_other(kw):
    assert attention(**kw) == BAD


def norm(**kw):
    a = dict(rows=4, width=64, dtype=1, codes_type=0, eps=1e-6, x=P, x_stride=64, out=2 * P, out_stride=64) | kw
    return tokens._functions().predecoder_rms_norm(None, tokens.NormArgs(**a))


@pytest.mark.parametrize("kw", [dict(out=P, out_stride=72), dict(x_stride=72, out=P), dict(sum=P, sum_stride=72), dict(residual=3 * P, residual_stride=72, sum=3 * P, sum_stride=64),
                                dict(residual=3 * P, residual_stride=64, out=3 * P, out_stride=128), dict(sum=2 * P, sum_stride=64)])
def test_norm_outputs_on_inputs_or_each_other(kw):
    """An input under another stride, or one place for both outputs."""
    assert norm(**kw) == BAD
