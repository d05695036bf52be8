"""Token operators: what a block of attention over the sites of detector volumes runs (include/predecoder_ops.h).

Thin ctypes binding, as for the pre-decoder: it checks that the tensors are what the kernels of libpredecoder.so
read and write, and passes their pointers, sizes and strides on.  Outputs are the caller's tensors; work is
enqueued on the current stream, or on `stream`.

A token is one site of one round of a volume.  Its place is a row (t, i, j, volume) of an int32 tensor ("sites");
volume < 0 marks a row that holds no token.

The operators are for inference: a tensor that asks for a gradient is refused while gradients are recorded.
"""
import ctypes
import struct

import torch

from . import (ACT_GELU_TANH, ACT_NONE, ACT_RELU, DTYPE_BF16, DTYPE_FP32, PD_OK, PredecoderError, lib)

__all__ = ["rms_norm", "matmul8", "rope", "attention", "attention_workspace", "volume_sites", "CODES_NONE",
           "CODES_E4M3", "CODES_INT8", "OPS_EXPORTS"]

CODES_NONE, CODES_E4M3, CODES_INT8 = 0, 1, 2
PREFIX_NONE = -(1 << 31)  # PD_PREFIX_NONE
_ACTS = {"none": ACT_NONE, "gelu": ACT_GELU_TANH, "relu": ACT_RELU}
_VALUES = {torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_FP32}
_CODES = {torch.float8_e4m3fn: CODES_E4M3, torch.int8: CODES_INT8}

# Every symbol declared in include/predecoder_ops.h.
OPS_EXPORTS = ("predecoder_rms_norm", "predecoder_matmul8", "predecoder_rope", "predecoder_attention_workspace",
               "predecoder_attention")

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class NormArgs(ctypes.Structure):
    _fields_ = [("rows", _i64), ("width", _i32), ("dtype", _i32), ("codes_type", _i32), ("eps", _f32),
                ("x", _vp), ("x_stride", _i64), ("residual", _vp), ("residual_stride", _i64), ("gain", _vp),
                ("sum", _vp), ("sum_stride", _i64), ("out", _vp), ("out_stride", _i64),
                ("codes", _vp), ("codes_stride", _i64), ("scales", _vp)]


class Matmul8Args(ctypes.Structure):
    _fields_ = [("M", _i64), ("N", _i32), ("K", _i32), ("codes_type", _i32), ("out_dtype", _i32), ("act", _i32),
                ("a", _vp), ("a_stride", _i64), ("a_scales", _vp), ("w", _vp), ("w_stride", _i64), ("w_scales", _vp),
                ("bias", _vp), ("out", _vp), ("out_stride", _i64)]


class RopeArgs(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("heads", _i32), ("head_dim", _i32), ("dtype", _i32), ("sections", _i32 * 3),
                ("interleaved", _i32), ("inverse", _i32), ("base", ctypes.c_double), ("sites", _vp),
                ("x", _vp), ("x_token_stride", _i64), ("x_head_stride", _i64),
                ("out", _vp), ("out_token_stride", _i64), ("out_head_stride", _i64)]


class AttentionArgs(ctypes.Structure):
    _fields_ = [("batch", _i32), ("heads", _i32), ("kv_heads", _i32), ("head_dim", _i32), ("n_q", _i32),
                ("n_k", _i32), ("scale", _f32), ("cap", _f32), ("causal", _i32), ("prefix", _i32)] + \
               [f for n in "qkv" for f in ((n, _vp), (n + "_batch_stride", _i64), (n + "_token_stride", _i64),
                                           (n + "_head_stride", _i64))] + \
               [("out", _vp), ("out_batch_stride", _i64), ("out_token_stride", _i64), ("out_head_stride", _i64),
                ("q_sites", _vp), ("q_sites_batch_stride", _i64), ("k_sites", _vp), ("k_sites_batch_stride", _i64),
                ("slopes", _vp), ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t)]


_fn = None


def _functions():
    """The library's functions, taking the structures above; looked up once."""
    global _fn
    if _fn is None:
        L = lib()
        for name, args in (("predecoder_rms_norm", NormArgs), ("predecoder_matmul8", Matmul8Args),
                           ("predecoder_rope", RopeArgs), ("predecoder_attention", AttentionArgs)):
            f = getattr(L, name)
            f.argtypes, f.restype = [_vp, ctypes.POINTER(args)], _i32
        L.predecoder_attention_workspace.argtypes = [ctypes.POINTER(AttentionArgs)]
        L.predecoder_attention_workspace.restype = ctypes.c_size_t
        _fn = L
    return _fn


# A small call's time is the host's: arguments are packed by struct (the structures' layout, native alignment), a third
# of the time that filling a ctypes structure takes, and handed over by functions that take the bytes.
_FORMAT = {_i64: "q", _i32: "i", _f32: "f", ctypes.c_double: "d", _vp: "P", ctypes.c_size_t: "N", _i32 * 3: "3i"}


def _packer(args):
    s = struct.Struct("@" + "".join(_FORMAT[f[1]] for f in args._fields_))
    assert s.size <= ctypes.sizeof(args) < s.size + 8  # (no padding at the end)
    return s.pack


_pack_norm, _pack_matmul8 = _packer(NormArgs), _packer(Matmul8Args)
_pack_rope, _pack_attention = _packer(RopeArgs), _packer(AttentionArgs)
_fast = {}


def _by_bytes(name):
    """The library's function `name`, taking packed arguments."""
    f = _fast.get(name)
    if f is None:
        f = lib()[name]
        work = name == "predecoder_attention_workspace"
        f.argtypes = [ctypes.c_char_p] if work else [_vp, ctypes.c_char_p]
        f.restype = ctypes.c_size_t if work else _i32
        _fast[name] = f
    return f


def _raw_stream(stream, index):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _call(name, args, stream, index):
    f = _by_bytes(name)
    if index == torch._C._cuda_getDevice():
        st = f(_raw_stream(stream, index), args)
    else:
        with torch.cuda.device(index):
            st = f(_raw_stream(stream, index), args)
    if st != PD_OK:
        raise PredecoderError(st, name)


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _index(t, what):
    """The index of the GPU that a tensor is on."""
    index = t.get_device()
    if index < 0:
        raise ValueError("%s must be a tensor on the GPU" % what)
    return index


def _lost_gradient(what):
    """Refuses a tensor that asks for a gradient while gradients are recorded."""
    if torch.is_grad_enabled():
        raise ValueError("%s asks for a gradient, which this operator does not give: call it under torch.no_grad()" % what)


def _matrix(t, what, shape, dtype, index):
    """Pointer and row stride of a device matrix with contiguous rows; zeros for None."""
    if t is None:
        return 0, 0
    if t.get_device() != index:
        raise ValueError("%s must be a tensor on GPU %d" % (what, index))
    if t.requires_grad:
        _lost_gradient(what)
    if t.dtype != dtype:
        raise ValueError("%s has type %s, expected %s" % (what, t.dtype, dtype))
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (what, tuple(t.shape), tuple(shape)))
    stride, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise ValueError("the rows of %s must be contiguous" % what)
    return t.data_ptr(), stride


def _vector(t, what, n, index):
    """Pointer of a contiguous device vector of n float32 values; 0 for None."""
    if t is None:
        return 0
    if t.get_device() != index:
        raise ValueError("%s must be a tensor on GPU %d" % (what, index))
    if t.requires_grad:
        _lost_gradient(what)
    if t.dtype != torch.float32 or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s must be a contiguous vector of %d float32 values" % (what, n))
    return t.data_ptr()


def rms_norm(x, gain=None, eps=1e-6, residual=None, sum_out=None, out=None, codes=None, scales=None, stream=None):
    """s = x + residual; y = s / sqrt(mean(s^2) + eps) * gain, over the rows of x [rows][width] (bf16 or float32).

    Writes what is given of: sum_out (s), out (y; both of x's type), codes [rows][width] (float8_e4m3fn or int8)
    with scales [rows]: y / scale rounded, scale = max |y| / 448 or / 127."""
    _need(x.dim() == 2, "x must be a matrix")
    dt, shape, dev = x.dtype, x.shape, _index(x, "x")
    _need(dt in _VALUES, "x must be bfloat16 or float32")
    _need((codes is None) == (scales is None), "codes and scales go together")
    _need(sum_out is not None or out is not None or codes is not None, "no output is given")
    rows, width = shape
    px, sx = _matrix(x, "x", shape, dt, dev)
    pr, sr = _matrix(residual, "residual", shape, dt, dev)
    ps, ss = _matrix(sum_out, "sum_out", shape, dt, dev)
    po, so = _matrix(out, "out", shape, dt, dev)
    ct = pc = sc = CODES_NONE
    if codes is not None:
        _need(codes.dtype in _CODES, "codes must be float8_e4m3fn or int8")
        ct = _CODES[codes.dtype]
        pc, sc = _matrix(codes, "codes", shape, codes.dtype, dev)
    _call("predecoder_rms_norm", _pack_norm(rows, width, _VALUES[dt], ct, eps, px, sx, pr, sr,
                                            _vector(gain, "gain", width, dev), ps, ss, po, so, pc, sc,
                                            _vector(scales, "scales", rows, dev)), stream, dev)


def matmul8(a, a_scales, w, w_scales, out, bias=None, act="none", stream=None):
    """out[m][n] = act(a_scales[m] w_scales[n] sum_k a[m][k] w[n][k] + bias[n]).

    a [M][K] and w [N][K]: 8-bit codes of one type (float8_e4m3fn or int8); scales and bias float32; act "none", "gelu" or
    "relu" (or an ACT_ constant); out [M][N] bfloat16 or float32."""
    _need(a.dim() == 2 and w.dim() == 2, "a and w must be matrices")
    dt, to, dev = a.dtype, out.dtype, _index(a, "a")
    _need(dt in _CODES, "a must be float8_e4m3fn or int8")
    _need(to in _VALUES, "out must be bfloat16 or float32")
    M, K = a.shape
    N = w.shape[0]
    pa, sa = _matrix(a, "a", (M, K), dt, dev)
    pw, sw = _matrix(w, "w", (N, K), dt, dev)
    po, so = _matrix(out, "out", (M, N), to, dev)
    _need(not isinstance(act, str) or act in _ACTS, "act must be none, gelu or relu")
    code = _ACTS[act] if isinstance(act, str) else int(act)
    _call("predecoder_matmul8", _pack_matmul8(M, N, K, _CODES[dt], _VALUES[to], code, pa, sa,
                                              _vector(a_scales, "a_scales", M, dev), pw, sw,
                                              _vector(w_scales, "w_scales", N, dev), _vector(bias, "bias", N, dev),
                                              po, so), stream, dev)


def _sites(t, what, n, index, batch=None):
    """Pointer and batch stride (in sites) of int32 sites [n][4] or, with a batch, [batch][n][4]."""
    if t.get_device() != index or t.dtype != torch.int32:
        raise ValueError("%s must be an int32 tensor on GPU %d" % (what, index))
    shape, s = t.shape, t.stride()
    if shape != (n, 4) and (batch is None or shape != (batch, n, 4)):
        raise ValueError("%s has shape %s, expected %s" % (what, tuple(shape), (n, 4)))
    if n and (s[-1] != 1 or (n > 1 and s[-2] != 4)):
        raise ValueError("%s must be contiguous" % what)
    if len(shape) == 2 or batch == 1:
        return t.data_ptr(), 0
    _need(s[0] % 4 == 0, "%s must hold whole sites from entry to entry" % what)
    return t.data_ptr(), s[0] // 4


def rope(x, sites, out, sections, base=10000.0, interleaved=False, inverse=False, stream=None):
    """Rotary positions: x [tokens][heads][head_dim] (bf16 or float32) turned by the tokens' sites into out (may be x).

    sections: pairs of a head that turn with the round, the row and the column; pair k of n turns by base^(-k/n) a step.
    A pair is values m and m + head_dim / 2, or 2 m and 2 m + 1 if interleaved.  inverse turns back."""
    dt, shape, dev = x.dtype, x.shape, _index(x, "x")
    _need(len(shape) == 3 and out.shape == shape, "x and out must be [tokens][heads][head_dim] of one shape")
    _need(dt in _VALUES and out.dtype == dt, "x and out must both be bfloat16 or both float32")
    _need(out.get_device() == dev, "x and out must be tensors on one GPU")
    if x.requires_grad:
        _lost_gradient("x")
    if out.requires_grad:
        _lost_gradient("out")
    n, H, D = shape
    xt, xh, x1 = x.stride()
    ot, oh, o1 = out.stride()
    _need(D <= 1 or (x1 == 1 and o1 == 1), "the rows of a head must be contiguous")
    s0, s1, s2 = sections
    _call("predecoder_rope", _pack_rope(n, H, D, _VALUES[dt], s0, s1, s2, bool(interleaved), bool(inverse), base,
                                        _sites(sites, "sites", n, dev)[0], x.data_ptr(), xt, xh, out.data_ptr(), ot, oh),
          stream, dev)


def _attention_args(q, k, v, out, q_sites, k_sites, scale, cap, slopes, causal, prefix):
    """The arguments of predecoder_attention for these tensors, without a workspace."""
    _need(q.dim() == 4 and k.dim() == 4, "q and k must be [batch][tokens][heads][head_dim]")
    shape, dev = q.shape, _index(q, "q")
    B, nq, H, D = shape
    _, nk, Hk, _ = k.shape
    fields = []
    for t, what, want in ((q, "q", shape), (k, "k", (B, nk, Hk, D)), (v, "v", (B, nk, Hk, D)), (out, "out", shape)):
        if t.get_device() != dev or t.dtype != torch.bfloat16 or t.shape != want:
            raise ValueError("%s must be a bfloat16 tensor %s on the GPU of q" % (what, tuple(want)))
        if t.requires_grad:
            _lost_gradient(what)
        sb, st, sh, one = t.stride()
        if one != 1 and D > 1:
            raise ValueError("the rows of a head must be contiguous in %s" % what)
        fields += (t.data_ptr(), sb, st, sh)
    _need((q_sites is None) == (k_sites is None), "q_sites and k_sites go together")
    pq = pk = bq = bk = 0
    if q_sites is not None:
        pq, bq = _sites(q_sites, "q_sites", nq, dev, B)
        pk, bk = _sites(k_sites, "k_sites", nk, dev, B)
    if scale is None:
        scale = D ** -0.5
    return (B, H, Hk, D, nq, nk, scale, cap, bool(causal),
            PREFIX_NONE if prefix is None else int(prefix), *fields, pq, bq, pk, bk,
            _vector(slopes, "slopes", H, dev))


def attention_workspace(q, k, v, out, q_sites=None, k_sites=None, scale=None, cap=0.0, slopes=None, causal=False,
                        prefix=None):
    """Bytes of workspace of attention() with these arguments."""
    a = _attention_args(q, k, v, out, q_sites, k_sites, scale, cap, slopes, causal, prefix)
    return _by_bytes("predecoder_attention_workspace")(_pack_attention(*a, 0, 0))


def attention(q, k, v, out, q_sites=None, k_sites=None, scale=None, cap=0.0, slopes=None, causal=False, prefix=None,
              workspace=None, stream=None):
    """Attention of q [batch][n_q][heads][head_dim] over k, v [batch][n_k][kv_heads][head_dim] into out (bf16).

    Scores scale q.k (scale None: head_dim^-1/2), capped by cap tanh(. / cap) if cap > 0, minus slopes[head] times the L1 distance
    of the sites; over the keys of the query's volume, with causal those of its own and earlier rounds or, unless prefix
    is None, of all rounds below prefix (for 0: the negative ones).  sites: [n][4] for all batch entries or
    [batch][n][4].  workspace: a device tensor of at least
    attention_workspace() bytes (needed with a raw stream handle; otherwise allocated here)."""
    a = _attention_args(q, k, v, out, q_sites, k_sites, scale, cap, slopes, causal, prefix)
    dev = q.get_device()
    ptr = 0
    if workspace is not None:
        _need(workspace.get_device() == dev and workspace.is_contiguous(),
              "workspace must be a contiguous tensor on the GPU of q")
        ptr, need = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    else:
        need = _by_bytes("predecoder_attention_workspace")(_pack_attention(*a, 0, 0))
        if need:
            if stream is None:
                workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
            else:
                _need(isinstance(stream, torch.cuda.Stream), "a raw stream handle needs a workspace from the caller")
                with torch.cuda.stream(stream):  # its memory goes back to the stream that uses it
                    workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
            ptr = workspace.data_ptr()
    _call("predecoder_attention", _pack_attention(*a, ptr, need), stream, dev)


def volume_sites(d, T, volume=0, first_round=0, layout="plaquette", device="cuda"):
    """The sites of a volume's activations in memory order: [T H H][4], H = d + 1 (plaquette layout) or d (paper layout)."""
    _need(layout in ("plaquette", "paper"), "layout must be plaquette or paper")
    H = d if layout == "paper" else d + 1
    t, i, j = torch.meshgrid(torch.arange(first_round, first_round + T, device=device), torch.arange(H, device=device),
                             torch.arange(H, device=device), indexing="ij")
    return torch.stack([t, i, j, torch.full_like(t, volume)], -1).reshape(-1, 4).to(torch.int32)
