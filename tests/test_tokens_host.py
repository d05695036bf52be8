"""Host-side checks of the token operators' C ABI (no kernel launches): the exported names, the layout of the argument
structures, refusals before any device call."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

import paper_2604_12841_amd as pdx
from conftest import ROOT
from paper_2604_12841_amd import tokens

HEADER = os.path.join(ROOT, "include", "predecoder_ops.h")
STRUCTS = {"pd_norm_args": tokens.NormArgs, "pd_matmul8_args": tokens.Matmul8Args, "pd_rope_args": tokens.RopeArgs,
           "pd_attention_args": tokens.AttentionArgs}


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(predecoder_\w+)\s*\(", text))
    assert names == set(tokens.OPS_EXPORTS)
    for n in names:
        assert hasattr(pdx.lib(), n)
    for n in ("rms_norm", "matmul8", "rope", "attention", "volume_sites"):
        assert callable(getattr(pdx, n)) and n in pdx.__all__


def test_structures_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    lines = []
    for name, s in STRUCTS.items():
        lines.append('printf("%%zu ", sizeof(%s));' % name)
        lines += ['printf("%%zu ", offsetof(%s, %s));' % (name, f[0]) for f in s._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "predecoder_ops.h"\nint main(void) {%s return 0;}' % "\n".join(lines))
    exe = str(tmp_path / "s")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-I" + os.path.dirname(HEADER), str(src), "-o", exe])
    want = []
    for s in STRUCTS.values():
        want += [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]
    assert [int(v) for v in subprocess.check_output([exe], text=True).split()] == want


P = 4096  # an aligned address that no call may touch


def call(name, args):
    return getattr(tokens._functions(), name)(None, args)


def norm(**kw):
    a = dict(rows=4, width=64, dtype=1, codes_type=0, eps=1e-6, x=P, x_stride=64, out=P, out_stride=64) | kw
    return call("predecoder_rms_norm", tokens.NormArgs(**a))


def matmul(**kw):
    a = dict(M=4, N=8, K=32, codes_type=2, out_dtype=1, act=0, a=P, a_stride=32, a_scales=P, w=P, w_stride=32, w_scales=P, out=P,
             out_stride=8) | kw
    return call("predecoder_matmul8", tokens.Matmul8Args(**a))


def rope(**kw):
    a = dict(tokens=4, heads=2, head_dim=32, dtype=1, sections=(8, 4, 4), interleaved=0, inverse=0, base=100.0, sites=P, x=P, x_token_stride=64,
             x_head_stride=32, out=P, out_token_stride=64, out_head_stride=32) | kw
    a["sections"] = (ctypes.c_int32 * 3)(*a["sections"])
    return call("predecoder_rope", tokens.RopeArgs(**a))


def attention(**kw):
    a = dict(batch=1, heads=4, kv_heads=2, head_dim=64, n_q=4, n_k=9, scale=0.1, cap=0.0, causal=0, prefix=0)
    for n in ("q", "k", "v", "out"):
        a |= {n: P, n + "_batch_stride": 4096, n + "_token_stride": 256, n + "_head_stride": 64}
    a |= dict(workspace=P, workspace_bytes=1 << 40)
    return call("predecoder_attention", tokens.AttentionArgs(**(a | kw)))


BAD, NO_FORM = pdx.PD_ERR_INVALID_ARG, pdx.PD_ERR_UNSUPPORTED


@pytest.mark.parametrize("want,kw", [(BAD, dict(rows=-1)), (BAD, dict(width=0)), (BAD, dict(dtype=2)), (BAD, dict(codes_type=3)), (BAD, dict(x=None)),
                                     (BAD, dict(out=None)), (BAD, dict(codes=P)), (BAD, dict(codes_type=1, codes=P, codes_stride=64)),
                                     (BAD, dict(codes_type=1, codes=P, codes_stride=63, scales=P)), (BAD, dict(out_stride=63)),
                                     (BAD, dict(eps=-1e-9)), (BAD, dict(x=P + 1)), (BAD, dict(gain=P + 2)), (NO_FORM, dict(width=32769, out_stride=40000)),
                                     (0, dict(rows=0))])
def test_norm_refusals(want, kw):
    assert norm(**kw) == want


@pytest.mark.parametrize("want,kw", [(BAD, dict(M=-1)), (BAD, dict(N=-1)), (BAD, dict(K=-1)), (BAD, dict(codes_type=0)), (BAD, dict(out_dtype=2)),
                                     (BAD, dict(act=3)), (BAD, dict(a=None)), (BAD, dict(w=None)), (BAD, dict(a_scales=None)), (BAD, dict(w_scales=None)),
                                     (BAD, dict(out=None)), (BAD, dict(out_stride=7)), (BAD, dict(out=P + 1)), (BAD, dict(bias=P + 1)),
                                     (NO_FORM, dict(K=131072, a_stride=131072, w_stride=131072)), (NO_FORM, dict(M=1 << 40)),
                                     (0, dict(M=0)), (0, dict(N=0, out_stride=0))])
def test_matmul_refusals(want, kw):
    assert matmul(**kw) == want


@pytest.mark.parametrize("want,kw", [(BAD, dict(tokens=-1)), (BAD, dict(heads=-1)), (BAD, dict(head_dim=31)), (BAD, dict(head_dim=0)), (BAD, dict(dtype=2)),
                                     (BAD, dict(sections=(8, 8, 1))), (BAD, dict(sections=(8, -1, 1))), (BAD, dict(base=0.0)), (BAD, dict(interleaved=2)),
                                     (BAD, dict(sections=(2147483647, 2147483647, 2))), (BAD, dict(inverse=-1)), (BAD, dict(sites=None)),
                                     (BAD, dict(sites=P + 4)), (BAD, dict(x=None)), (BAD, dict(out=P + 1)), (NO_FORM, dict(head_dim=258)),
                                     (NO_FORM, dict(tokens=1 << 41)), (0, dict(tokens=0)), (0, dict(heads=0))])
def test_rope_refusals(want, kw):
    assert rope(**kw) == want


@pytest.mark.parametrize("want,kw", [(BAD, dict(batch=-1)), (BAD, dict(heads=3)), (BAD, dict(kv_heads=0)), (BAD, dict(head_dim=0)), (NO_FORM, dict(head_dim=12)),
                                     (NO_FORM, dict(head_dim=136)), (BAD, dict(n_q=-1)), (BAD, dict(n_k=-1)), (BAD, dict(scale=float("nan"))),
                                     (BAD, dict(cap=-1.0)), (BAD, dict(causal=2)), (BAD, dict(prefix=1)), (BAD, dict(causal=1)), (BAD, dict(slopes=P)),
                                     (BAD, dict(q_sites=P)), (BAD, dict(k_sites=P)), (BAD, dict(q_sites=P + 8, k_sites=P)), (BAD, dict(q=None)),
                                     (BAD, dict(k=None)), (BAD, dict(out=None)), (NO_FORM, dict(q=P + 2)), (NO_FORM, dict(k_token_stride=132)),
                                     (NO_FORM, dict(heads=130, kv_heads=2)), (NO_FORM, dict(batch=65536)), (NO_FORM, dict(n_q=2147483647)),
                                     (0, dict(batch=0)), (0, dict(n_q=0)), (0, dict(heads=0))])
def test_attention_refusals(want, kw):
    assert attention(**kw) == want


def test_workspace_is_asked_for_before_the_call():
    a = dict(batch=1, heads=8, kv_heads=2, head_dim=64, n_q=1, n_k=100000, scale=0.1)
    need = tokens._functions().predecoder_attention_workspace(tokens.AttentionArgs(**a))
    if need:
        assert attention(heads=8, n_q=1, n_k=100000, workspace=None) == BAD
        assert attention(heads=8, n_q=1, n_k=100000, workspace_bytes=need - 1) == BAD
        assert attention(heads=8, n_q=1, n_k=100000, workspace=P + 4) == BAD
    assert tokens._functions().predecoder_attention_workspace(tokens.AttentionArgs(**(a | dict(head_dim=12)))) == 0
    assert tokens._functions().predecoder_attention_workspace(None) == 0


def test_sizes_whose_products_pass_64_bits():
    """kv_heads x batch x rows x bytes of a row = 2^64: refused, the plan's divisions included."""
    many = dict(batch=32768, heads=32768, kv_heads=32768, head_dim=128, n_q=1 << 25, n_k=64)
    assert attention(**many) == NO_FORM
    assert tokens._functions().predecoder_attention_workspace(tokens.AttentionArgs(scale=0.1, **many)) == 0


def test_work_items_are_counted_as_they_are_launched():
    """4095 x 4097 = 2^24 - 1 items are launched as 2^24 workgroups of 256 threads: one thread too many for a grid."""
    assert attention(batch=4097, heads=4095, kv_heads=4095, n_q=128, n_k=64) == NO_FORM
    # (many heads, not many: the last size that has a form asks for its workspace and no less)
    assert attention(batch=4096, heads=4095, kv_heads=4095, n_q=128, n_k=300, q_sites=P, k_sites=P, workspace=None) == BAD


def test_rotary_work_items_stay_within_64_bits():
    assert rope(tokens=1 << 40, heads=1 << 20, head_dim=256) == NO_FORM
