"""Host-side checks of the C ABI of the 8-bit cache, attention over it, and linear attention (no kernel launches)."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2604_12841_amd as pdx
from conftest import ROOT
from paper_2604_12841_amd import tokens

HEADER = os.path.join(ROOT, "include", "predecoder_ops.h")
P = 4096  # an aligned address that no call may touch
BAD, NO_FORM = pdx.PD_ERR_INVALID_ARG, pdx.PD_ERR_UNSUPPORTED
CACHE = dict(batch=2, kv_heads=2, head_dim=64, capacity=100, codes_type=1, codes=P, scales=P, cache_sites=P)


def test_structures_match_the_header(tmp_path):
    """Their first members are pd_cache's, one after the other."""
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    names = {"cache_sites": "cache.sites"} | {n: "cache." + n for n in ("batch", "kv_heads", "head_dim", "capacity", "codes_type", "codes", "scales")}
    lines, want = [], []
    for name, s, held in (("pd_cache_args", tokens.CacheArgs, True), ("pd_attention8_args", tokens.Attention8Args, True),
                          ("pd_linear_attention_args", tokens.LinearAttentionArgs, False)):
        lines.append('printf("%%zu ", sizeof(%s));' % name)
        lines += ['printf("%%zu ", offsetof(%s, %s));' % (name, names.get(f[0], f[0]) if held else f[0]) for f in s._fields_]
        want += [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "predecoder_ops.h"\nint main(void) {%s return 0;}' % "\n".join(lines))
    exe = str(tmp_path / "s")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-I" + os.path.dirname(HEADER), str(src), "-o", exe])
    assert [int(v) for v in subprocess.check_output([exe], text=True).split()] == want


def cache(name, **kw):
    a = CACHE | dict(tokens=10, dtype=1, at=P, sites=P, sites_batch_stride=10)
    for n in "kv":
        a |= {n: P if n == "k" else 2 * P, n + "_batch_stride": 4096, n + "_token_stride": 128, n + "_head_stride": 64}
    return getattr(tokens._functions(), "predecoder_cache_" + name)(None, tokens.CacheArgs(**(a | kw)))


COMMON = [(BAD, dict(batch=-1)), (BAD, dict(kv_heads=-1)), (BAD, dict(capacity=-1)), (BAD, dict(head_dim=0)), (BAD, dict(codes_type=0)), (BAD, dict(codes_type=3)),
          (NO_FORM, dict(head_dim=24)), (NO_FORM, dict(head_dim=144)), (NO_FORM, dict(batch=65536)), (NO_FORM, dict(kv_heads=65536)), (BAD, dict(codes=None)),
          (BAD, dict(scales=None)), (BAD, dict(cache_sites=None)), (BAD, dict(codes=P + 8)), (BAD, dict(scales=P + 2)), (BAD, dict(cache_sites=P + 4))]


@pytest.mark.parametrize("want,kw", COMMON + [(BAD, dict(tokens=-1)), (BAD, dict(tokens=101)), (BAD, dict(dtype=2)), (BAD, dict(at=None)), (BAD, dict(at=P + 4)),
                                              (BAD, dict(k=None)), (BAD, dict(v=None)), (BAD, dict(sites=P + 8)), (BAD, dict(k=P + 1)),
                                              (NO_FORM, dict(batch=65535, kv_heads=65535)), (0, dict(tokens=0)), (0, dict(batch=0)), (0, dict(kv_heads=0)),
                                              (0, dict(capacity=0, tokens=0, codes=None))])
@pytest.mark.parametrize("name", ["write", "read"])
def test_cache_refusals(name, want, kw):
    assert cache(name, **kw) == want


def test_cache_outputs_apart():
    """Rows that a read would write twice; the same strides are fine to read from."""
    for kw in (dict(k_token_stride=64), dict(v_head_stride=32), dict(k_batch_stride=0), dict(v=P), dict(sites_batch_stride=9)):
        assert cache("read", **kw) == BAD
    assert cache("write", sites=None) == BAD
    assert cache("read", sites=None, tokens=0) == 0


def attention8(**kw):
    a = CACHE | dict(heads=4, n_q=3, scale=0.1, cap=0.0, causal=0, prefix=0, q_sites=P, workspace=P, workspace_bytes=1 << 40)
    for n in ("q", "out"):
        a |= {n: P if n == "q" else 2 * P, n + "_batch_stride": 4096, n + "_token_stride": 256, n + "_head_stride": 64}
    return tokens._functions().predecoder_attention8(None, tokens.Attention8Args(**(a | kw)))


@pytest.mark.parametrize("want,kw", COMMON + [(BAD, dict(heads=-2)), (BAD, dict(heads=3)), (BAD, dict(n_q=-1)), (BAD, dict(scale=float("nan"))), (BAD, dict(cap=-1.0)),
                                              (BAD, dict(cap=float("inf"))), (BAD, dict(causal=2)), (BAD, dict(prefix=1)), (BAD, dict(causal=1, prefix=-1)),
                                              (BAD, dict(q=None)), (BAD, dict(out=None)), (BAD, dict(q_sites=None)), (BAD, dict(q_sites=P + 8)),
                                              (BAD, dict(slopes=P + 2)), (BAD, dict(out=P)), (NO_FORM, dict(q=P + 2)), (NO_FORM, dict(out_token_stride=260)),
                                              (BAD, dict(out_token_stride=64)), (NO_FORM, dict(heads=130)), (NO_FORM, dict(n_q=2147483647)),
                                              (BAD, dict(kv_heads=0)), (0, dict(n_q=0)), (0, dict(batch=0)), (0, dict(heads=0))])
def test_attention8_refusals(want, kw):
    assert attention8(**kw) == want


def linear(**kw):
    a = dict(batch=2, heads=4, kv_heads=2, head_dim=64, n=6, per_round=2, scale=0.1, workspace=P, workspace_bytes=1 << 40)
    for m, n in enumerate(("q", "k", "v", "out")):
        a |= {n: (m + 1) * P, n + "_batch_stride": 4096, n + "_token_stride": 256, n + "_head_stride": 64}
    return tokens._functions().predecoder_linear_attention(None, tokens.LinearAttentionArgs(**(a | kw)))


@pytest.mark.parametrize("want,kw", [(BAD, dict(batch=-1)), (BAD, dict(heads=3)), (BAD, dict(kv_heads=0)), (BAD, dict(heads=-4)), (BAD, dict(n=-1)),
                                     (BAD, dict(per_round=0)), (BAD, dict(head_dim=0)), (NO_FORM, dict(head_dim=12)), (NO_FORM, dict(head_dim=136)),
                                     (BAD, dict(scale=float("inf"))), (BAD, dict(q=None)), (BAD, dict(k=None)), (BAD, dict(v=None)), (BAD, dict(out=None)),
                                     (BAD, dict(out=P)), (BAD, dict(out=2 * P)), (BAD, dict(out=3 * P)), (BAD, dict(slopes=P + 2)), (BAD, dict(lengths=P + 2)),
                                     (BAD, dict(state=P + 4)), (BAD, dict(state_out=P + 4)), (NO_FORM, dict(k=2 * P + 8)), (NO_FORM, dict(v_head_stride=60)),
                                     (BAD, dict(out_token_stride=128)), (NO_FORM, dict(heads=130)), (NO_FORM, dict(n=2147483647)),
                                     (NO_FORM, dict(batch=65535, heads=65535, kv_heads=65535)), (0, dict(batch=0)), (0, dict(heads=0, kv_heads=0))])
def test_linear_refusals(want, kw):
    assert linear(**kw) == want


def test_linear_states_apart():
    """state_out is state itself or lies apart from it, also where no token comes; without a query head no state is handed on."""
    size = 2 * 2 * 64 * 64 * 4  # of the batch, key heads and head size of linear()
    for n in (0, 1, 5):
        for off in (64, size - 16):
            assert linear(n=n, state=16 * P, state_out=16 * P + off) == BAD
            assert linear(n=n, state=16 * P + off, state_out=16 * P) == BAD
    for state in (None, 16 * P):
        assert linear(heads=0, state=state, state_out=32 * P) == BAD
    assert linear(heads=0, state=16 * P) == 0 and linear(heads=0, kv_heads=0, state=16 * P, state_out=16 * P) == 0


LONG = dict(batch=1, heads=2, kv_heads=2, head_dim=64, n=100000, per_round=4, scale=0.1)


def test_workspaces_are_asked_for_before_the_call():
    f = tokens._functions()
    need = f.predecoder_linear_attention_workspace(tokens.LinearAttentionArgs(**LONG))
    assert need > 0
    for kw in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 4)):
        assert linear(**(LONG | kw)) == BAD
    many = dict(batch=1, capacity=100000, n_q=1)
    need = f.predecoder_attention8_workspace(tokens.Attention8Args(**(CACHE | dict(heads=4, scale=0.1) | many)))
    assert need > 0
    for kw in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 4)):
        assert attention8(**(many | kw)) == BAD
    # by the sizes alone: no pointer is followed
    assert need == f.predecoder_attention8_workspace(tokens.Attention8Args(**(CACHE | dict(heads=4, scale=0.1, codes=None, scales=None, cache_sites=None) | many)))
    for n, s in (("attention8", tokens.Attention8Args), ("linear_attention", tokens.LinearAttentionArgs)):
        w = getattr(f, "predecoder_%s_workspace" % n)
        assert w(None) == 0 and w(s(head_dim=12)) == 0
        assert getattr(f, "predecoder_" + n)(None, None) == BAD
    assert f.predecoder_cache_write(None, None) == BAD and f.predecoder_cache_read(None, None) == BAD


def test_sizes_at_the_end_of_their_range():
    """Plans of the largest sizes: no overflow, no division by zero (the host sanitizers run this too)."""
    big = 2147483647
    f = tokens._functions()
    for kw in (dict(n=big // 2, per_round=1), dict(n=big // 2, per_round=big), dict(n=1, per_round=big), dict(n=0), dict(n=100, per_round=33, heads=64, kv_heads=1),
               dict(batch=65535, heads=2, kv_heads=2), dict(head_dim=128, n=1 << 29), dict(batch=big, heads=1, kv_heads=1, n=1)):
        f.predecoder_linear_attention_workspace(tokens.LinearAttentionArgs(**(dict(LONG, heads=1, kv_heads=1) | kw)))
    for kw in (dict(capacity=big, n_q=1), dict(capacity=big, n_q=1 << 24), dict(capacity=0, n_q=5), dict(capacity=1, n_q=1), dict(batch=65535, n_q=64, capacity=big)):
        f.predecoder_attention8_workspace(tokens.Attention8Args(**(CACHE | dict(heads=4, scale=0.1) | kw)))
