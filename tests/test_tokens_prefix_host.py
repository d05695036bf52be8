"""Host-side checks of attention's prefix (no kernel launches)."""
import os
import re

from conftest import ROOT
from paper_2604_12841_amd import tokens


def workspace(**kw):
    a = dict(batch=1, heads=8, kv_heads=2, head_dim=64, n_q=1, n_k=100000, scale=0.1, causal=1) | kw
    return tokens._functions().predecoder_attention_workspace(tokens.AttentionArgs(**a))


def test_no_prefix():
    need = workspace(prefix=0)
    assert need > 0
    assert workspace(prefix=tokens.PREFIX_NONE) == need and workspace(prefix=tokens.PREFIX_NONE, causal=0) == need
    for bad in (-1, tokens.PREFIX_NONE + 1):
        assert workspace(prefix=bad) == 0  # refused
    text = open(os.path.join(ROOT, "include", "predecoder_ops.h")).read()
    assert re.search(r"#define PD_PREFIX_NONE INT32_MIN\b", text) and tokens.PREFIX_NONE == -(1 << 31)
