"""Token operators: what a block of attention over the sites of detector volumes runs (include/predecoder_ops.h).

Thin ctypes binding, as for the pre-decoder: it checks that the tensors are what the kernels of libpredecoder.so
read and write, and passes their pointers, sizes and strides on.  Outputs are the caller's tensors; work is
enqueued on the current stream, or on `stream`.

A token is one site of one round of a volume.  Its place is a row (t, i, j, volume) of an int32 tensor ("sites");
volume < 0 marks a row that holds no token.
"""
import ctypes

import torch

from . import (ACT_GELU_TANH, ACT_NONE, ACT_RELU, DTYPE_BF16, DTYPE_FP32, PD_OK, PredecoderError, lib)

__all__ = ["rms_norm", "matmul8", "rope", "attention", "attention_workspace", "volume_sites", "CODES_NONE",
           "CODES_E4M3", "CODES_INT8", "OPS_EXPORTS"]

CODES_NONE, CODES_E4M3, CODES_INT8 = 0, 1, 2
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
    """The library's functions with their argument types, looked up once."""
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


def _raw_stream(stream, device):
    if stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _call(name, args, stream, device):
    f = getattr(_functions(), name)
    if device.index == torch.cuda.current_device():
        st = f(_raw_stream(stream, device), args)
    else:
        with torch.cuda.device(device):
            st = f(_raw_stream(stream, device), args)
    if st != PD_OK:
        raise PredecoderError(st, name)


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _matrix(t, what, shape, dtype, device):
    """Pointer and row stride of a device matrix with contiguous rows; (None, 0) for None."""
    if t is None:
        return None, 0
    if t.device != device or not t.is_cuda:
        raise ValueError("%s must be a tensor on %s" % (what, device if device.type == "cuda" else "the GPU"))
    if t.dtype != dtype:
        raise ValueError("%s has type %s, expected %s" % (what, t.dtype, dtype))
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (what, tuple(t.shape), tuple(shape)))
    s = t.stride()
    if s[1] != 1 and shape[1] > 1:
        raise ValueError("the rows of %s must be contiguous" % what)
    return t.data_ptr(), s[0]


def _vector(t, what, n, dtype, device):
    """Pointer of a contiguous device vector of n values; None for None."""
    if t is None:
        return None
    if t.device != device or not t.is_cuda:
        raise ValueError("%s must be a tensor on %s" % (what, device if device.type == "cuda" else "the GPU"))
    if t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError("%s must be a contiguous vector of %d values of type %s" % (what, n, dtype))
    return t.data_ptr()


def rms_norm(x, gain=None, eps=1e-6, residual=None, sum_out=None, out=None, codes=None, scales=None, stream=None):
    """s = x + residual; y = s / sqrt(mean(s^2) + eps) * gain, over the rows of x [rows][width] (bf16 or float32).

    Writes what is given of: sum_out (s), out (y; both of x's type), codes [rows][width] (float8_e4m3fn or int8)
    with scales [rows]: y / scale rounded, scale = max |y| / 448 or / 127."""
    _need(x.dim() == 2, "x must be a matrix")
    _need(x.dtype in _VALUES, "x must be bfloat16 or float32")
    _need(codes is None or codes.dtype in _CODES, "codes must be float8_e4m3fn or int8")
    _need((codes is None) == (scales is None), "codes and scales go together")
    _need(sum_out is not None or out is not None or codes is not None, "no output is given")
    shape, dt, dev = x.shape, x.dtype, x.device
    rows, width = shape
    px, sx = _matrix(x, "x", shape, dt, dev)
    pr, sr = _matrix(residual, "residual", shape, dt, dev)
    ps, ss = _matrix(sum_out, "sum_out", shape, dt, dev)
    po, so = _matrix(out, "out", shape, dt, dev)
    ct = CODES_NONE if codes is None else _CODES[codes.dtype]
    pc, sc = _matrix(codes, "codes", shape, codes.dtype if codes is not None else None, dev)
    a = NormArgs(rows, width, _VALUES[dt], ct, eps, px, sx, pr, sr, _vector(gain, "gain", width, torch.float32, dev), ps,
                 ss, po, so, pc, sc, _vector(scales, "scales", rows, torch.float32, dev))
    _call("predecoder_rms_norm", a, stream, dev)


def matmul8(a, a_scales, w, w_scales, out, bias=None, act="none", stream=None):
    """out[m][n] = act(a_scales[m] w_scales[n] sum_k a[m][k] w[n][k] + bias[n]).

    a [M][K] and w [N][K]: 8-bit codes of one type (float8_e4m3fn or int8); scales and bias float32; act "none", "gelu" or
    "relu" (or an ACT_ constant); out [M][N] bfloat16 or float32."""
    _need(a.dim() == 2 and w.dim() == 2, "a and w must be matrices")
    _need(a.dtype in _CODES, "a must be float8_e4m3fn or int8")
    _need(out.dtype in _VALUES, "out must be bfloat16 or float32")
    M, K = a.shape
    N = w.shape[0]
    dev = a.device
    pa, sa = _matrix(a, "a", (M, K), a.dtype, dev)
    pw, sw = _matrix(w, "w", (N, K), a.dtype, dev)
    po, so = _matrix(out, "out", (M, N), out.dtype, dev)
    code = _ACTS[act] if isinstance(act, str) else int(act)
    args = Matmul8Args(M, N, K, _CODES[a.dtype], _VALUES[out.dtype], code, pa, sa,
                       _vector(a_scales, "a_scales", M, torch.float32, dev), pw, sw,
                       _vector(w_scales, "w_scales", N, torch.float32, dev),
                       _vector(bias, "bias", N, torch.float32, dev), po, so)
    _call("predecoder_matmul8", args, stream, dev)


def _sites(t, what, n, device, batch=None):
    """Pointer and batch stride (in sites) of int32 sites [n][4] or, with a batch, [batch][n][4]."""
    _need(t.is_cuda and t.device == device, "%s must be a tensor on %s" % (what, device))
    _need(t.dtype == torch.int32, "%s must be int32" % what)
    shape = tuple(t.shape)
    _need(shape == (n, 4) or (batch is not None and shape == (batch, n, 4)),
          "%s has shape %s, expected %s" % (what, shape, (n, 4)))
    s = t.stride()
    _need(n == 0 or (s[-1] == 1 and (n == 1 or s[-2] == 4)), "%s must be contiguous" % what)
    if t.dim() == 2:
        return t.data_ptr(), 0
    _need(batch == 1 or s[0] % 4 == 0, "%s must hold whole sites from entry to entry" % what)
    return t.data_ptr(), s[0] // 4 if batch > 1 else 0


def rope(x, sites, out, sections, base=10000.0, interleaved=False, inverse=False, stream=None):
    """Rotary positions: x [tokens][heads][head_dim] (bf16 or float32) turned by the tokens' sites into out (may be x).

    sections: pairs of a head that turn with the round, the row and the column; pair k of n turns by base^(-k/n) a step.
    A pair is values m and m + head_dim / 2, or 2 m and 2 m + 1 if interleaved.  inverse turns back."""
    _need(x.dim() == 3 and out.dim() == 3, "x and out must be [tokens][heads][head_dim]")
    _need(x.dtype in _VALUES and out.dtype == x.dtype, "x and out must both be bfloat16 or both float32")
    _need(x.shape == out.shape, "x and out differ in shape")
    _need(x.is_cuda and out.device == x.device, "x and out must be tensors on one GPU")
    n, H, D = x.shape
    sx, so = x.stride(), out.stride()
    _need(D <= 1 or (sx[2] == 1 and so[2] == 1), "the rows of a head must be contiguous")
    ps, _ = _sites(sites, "sites", n, x.device)
    a = RopeArgs(n, H, D, _VALUES[x.dtype], (_i32 * 3)(*sections), int(interleaved), int(inverse), base, ps,
                 x.data_ptr(), sx[0], sx[1], out.data_ptr(), so[0], so[1])
    _call("predecoder_rope", a, stream, x.device)


def _attention_args(q, k, v, out, q_sites, k_sites, scale, cap, slopes, causal, prefix):
    """The arguments of predecoder_attention for these tensors, without a workspace."""
    _need(q.dim() == 4 and k.dim() == 4, "q and k must be [batch][tokens][heads][head_dim]")
    B, nq, H, D = q.shape
    nk, Hk = k.shape[1], k.shape[2]
    dev = q.device
    fields = []
    for t, what, shape in ((q, "q", q.shape), (k, "k", (B, nk, Hk, D)), (v, "v", (B, nk, Hk, D)), (out, "out", q.shape)):
        if not t.is_cuda or t.device != dev or t.dtype != torch.bfloat16 or t.shape != shape:
            raise ValueError("%s must be a bfloat16 tensor %s on the GPU of q" % (what, tuple(shape)))
        s = t.stride()
        if s[3] != 1 and D > 1:
            raise ValueError("the rows of a head must be contiguous in %s" % what)
        fields += [t.data_ptr(), s[0], s[1], s[2]]
    _need((q_sites is None) == (k_sites is None), "q_sites and k_sites go together")
    pq = pk = None
    bq = bk = 0
    if q_sites is not None:
        pq, bq = _sites(q_sites, "q_sites", nq, dev, B)
        pk, bk = _sites(k_sites, "k_sites", nk, dev, B)
    if scale is None:
        scale = D ** -0.5
    return AttentionArgs(B, H, Hk, D, nq, nk, scale, cap, int(causal), int(prefix), *fields, pq, bq, pk, bk,
                         _vector(slopes, "slopes", H, torch.float32, dev), None, 0)


def attention_workspace(q, k, v, out, q_sites=None, k_sites=None, scale=None, cap=0.0, slopes=None, causal=False,
                        prefix=0):
    """Bytes of workspace of attention() with these arguments."""
    a = _attention_args(q, k, v, out, q_sites, k_sites, scale, cap, slopes, causal, prefix)
    return int(_functions().predecoder_attention_workspace(a))


def attention(q, k, v, out, q_sites=None, k_sites=None, scale=None, cap=0.0, slopes=None, causal=False, prefix=0,
              workspace=None, stream=None):
    """Attention of q [batch][n_q][heads][head_dim] over k, v [batch][n_k][kv_heads][head_dim] into out (bf16).

    Scores scale q.k (scale None: head_dim^-1/2), capped by cap tanh(. / cap) if cap > 0, minus slopes[head] times the L1 distance
    of the sites; over the keys of the query's volume, with causal those of its own and earlier rounds or of rounds
    below prefix.  sites: [n][4] for all batch entries or [batch][n][4].  workspace: a device tensor of at least
    attention_workspace() bytes (needed with a raw stream handle; otherwise allocated here)."""
    a = _attention_args(q, k, v, out, q_sites, k_sites, scale, cap, slopes, causal, prefix)
    need = _functions().predecoder_attention_workspace(a)
    if workspace is not None:
        _need(workspace.is_cuda and workspace.device == q.device and workspace.is_contiguous(),
              "workspace must be a contiguous tensor on the GPU of q")
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    elif need:
        if stream is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        else:
            _need(isinstance(stream, torch.cuda.Stream), "a raw stream handle needs a workspace from the caller")
            with torch.cuda.stream(stream):  # its memory goes back to the stream that uses it
                workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        a.workspace, a.workspace_bytes = workspace.data_ptr(), need
    _call("predecoder_attention", a, stream, q.device)


def volume_sites(d, T, volume=0, first_round=0, layout="plaquette", device="cuda"):
    """The sites of a volume's activations in memory order: [T H H][4], H = d + 1 (plaquette layout) or d (paper layout)."""
    H = d if layout == "paper" else d + 1
    t, i, j = torch.meshgrid(torch.arange(first_round, first_round + T, device=device), torch.arange(H, device=device),
                             torch.arange(H, device=device), indexing="ij")
    return torch.stack([t, i, j, torch.full_like(t, volume)], -1).reshape(-1, 4).to(torch.int32)
