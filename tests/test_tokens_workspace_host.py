"""Host-side checks of what attention's workspace is asked for with (no kernel launches)."""
import pytest

import paper_2604_12841_amd as pdx
from paper_2604_12841_amd import tokens

P = 4096  # an aligned address that no call may touch


def args(**kw):
    a = dict(batch=2, heads=8, kv_heads=2, head_dim=64, n_q=1, n_k=100000, scale=0.1)
    for n in ("q", "k", "v", "out"):
        a |= {n: P, n + "_batch_stride": 1 << 24, n + "_token_stride": 512, n + "_head_stride": 64}
    return tokens.AttentionArgs(**(a | kw))


def need(**kw):
    return tokens._functions().predecoder_attention_workspace(args(**kw))


SITES = dict(q_sites=P, k_sites=P)


@pytest.mark.parametrize("kw", [{}, SITES, SITES | dict(k_sites_batch_stride=100000), SITES | dict(n_q=300, n_k=300)])
def test_a_byte_less_is_refused(kw):
    n = need(**kw)
    assert n > 0
    f = tokens._functions().predecoder_attention
    assert f(None, args(workspace=P, workspace_bytes=n - 1, **kw)) == pdx.PD_ERR_INVALID_ARG
    assert f(None, args(workspace=P + 4, workspace_bytes=n, **kw)) == pdx.PD_ERR_INVALID_ARG
    assert f(None, args(workspace=None, workspace_bytes=n, **kw)) == pdx.PD_ERR_INVALID_ARG


def test_what_the_size_goes_by():
    """Whether there are sites, and whether each entry has a list of its own; not where anything lies."""
    plain, one, each = need(), need(**SITES), need(k_sites_batch_stride=100000, **SITES)
    assert plain < one < each
    assert one == need(k_sites=64 * P) == need(k_sites=P, q=None, k=None, v=None, out=None, slopes=None)
    # asked without the sites that the call will have, the size is too small, and the call refused
    a = args(workspace=P, workspace_bytes=plain, **SITES)
    assert tokens._functions().predecoder_attention(None, a) == pdx.PD_ERR_INVALID_ARG
