"""The operators of a training step around the optimizer, on tensors.

``embed`` / ``embed_grad``              a token table's rows, and its gradient
``qk_norm_rope`` / ``qk_norm_rope_grad``  norms of queries and keys per head with the
                                        position rotation, and their backward pass
``act_pack`` / ``act_unpack``           an activation held in 8 bits for the backward pass
``weight_grad``                         a weight matrix's gradient from such an activation

As in the rest of the binding: argument checks and marshalling only, the work is
the native library's; calls are asynchronous on ``stream`` (default: torch's
current stream), results are fresh tensors unless ``out`` is given, and an error
of the library raises HimuonError. Tensors are float32 or bfloat16.
"""
from __future__ import annotations

import ctypes

from . import OK, HimuonError, _dtype_code, _keep_alive, lib

I32, I64 = 0, 1              # himuon_index_t
MAX_HEAD_DIM = 512           # HIMUON_MAX_HEAD_DIM
ACT_GROUP = 32               # HIMUON_ACT_GROUP: tokens of a column that share an exponent

_i64, _vp, _sz, _f, _int = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float, ctypes.c_int


class Heads(ctypes.Structure):
    """himuon_heads_t"""
    _fields_ = [("ptr", _vp), ("stride_batch", _i64), ("stride_seq", _i64), ("stride_head", _i64)]


class Qk(ctypes.Structure):
    """himuon_qk_t"""
    _fields_ = [("batch", _i64), ("seq", _i64), ("q_heads", ctypes.c_int32), ("k_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("gain_dtype", ctypes.c_int32), ("index", ctypes.c_int32),
                ("q_gain", _vp), ("k_gain", _vp), ("cos_table", _vp), ("sin_table", _vp), ("table_rows", _i64),
                ("positions", _vp), ("eps", _f)]


def declare(L):
    """Argument types of the operators' entry points (called once, as the library is loaded)."""
    heads = ctypes.POINTER(Heads)
    L.himuon_embed.argtypes = [_i64, _vp, _int, _i64, _i64, _vp, _i64, _vp, _i64, _f, _int, _vp]
    L.himuon_embed_grad_workspace_size.argtypes = [_i64, _i64, _i64]
    L.himuon_embed_grad.argtypes = [_i64, _vp, _int, _i64, _i64, _vp, _i64, _int, _vp, _i64, _int, _f, _int, _vp, _sz, _vp]
    L.himuon_qk_norm_rope.argtypes = [ctypes.POINTER(Qk)] + [heads] * 4 + [_vp]
    L.himuon_qk_norm_rope_grad_workspace_size.argtypes = [_i64, _i64, _i64]
    L.himuon_qk_norm_rope_grad.argtypes = [ctypes.POINTER(Qk)] + [heads] * 6 + [_vp, _vp, _vp, _sz, _vp]
    L.himuon_act_pack.argtypes = [_i64, _i64, _vp, _i64, _int, _vp, _vp, _vp]
    L.himuon_act_unpack.argtypes = [_i64, _i64, _vp, _vp, _vp, _i64, _int, _vp]
    L.himuon_weight_grad_workspace_size.argtypes = [_i64, _i64, _i64, _vp, _i64, _int]
    L.himuon_weight_grad.argtypes = [_i64, _i64, _i64, _vp, _i64, _int, _vp, _vp, _vp, _i64, _int, _int, _vp, _sz, _vp]
    for name in ("embed", "embed_grad", "qk_norm_rope", "qk_norm_rope_grad", "act_pack", "act_unpack", "weight_grad"):
        getattr(L, "himuon_" + name).restype = _int
    for name in ("embed_grad", "qk_norm_rope_grad", "weight_grad"):
        getattr(L, f"himuon_{name}_workspace_size").restype = _sz


# ------------------------------------------------------------------ shared checks

_INDEX = {}


def _torch():
    import torch
    if not _INDEX:
        _INDEX.update({torch.int32: I32, torch.int64: I64})
    return torch


def _index_code(t):
    code = _INDEX.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported index type {t.dtype}; expected int32 or int64")
    return code


def _matrix(t, what):
    """Checks a row-major CUDA matrix; its leading dimension."""
    if t.dim() != 2 or not t.is_cuda or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{what} must be a 2-D row-major CUDA tensor")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _same_device(dev, *tensors):
    for t in tensors:
        if t is not None and t.device != dev:
            raise ValueError("tensors must be on one device")


class _Call:
    """The stream of a call, its device made current, and the tensors allocated for it."""

    __slots__ = ("dev", "stream", "raw", "fresh", "prev")

    def __init__(self, dev, stream):
        torch = _torch()
        self.dev, self.stream, self.fresh = dev, stream, []
        # the default stream has no handle that names its device
        cur = torch._C._cuda_getDevice()
        self.prev = cur if cur != dev.index else None
        if self.prev is not None:
            torch.cuda.set_device(dev)
        self.raw = (torch._C._cuda_getCurrentRawStream(dev.index) if stream is None else stream.cuda_stream) or None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        if self.stream is not None:
            _keep_alive(self.fresh, self.stream, self.dev)
        if self.prev is not None:
            _torch().cuda.set_device(self.prev)

    def empty(self, shape, dtype):
        t = _torch().empty(shape, dtype=dtype, device=self.dev)
        self.fresh.append(t)
        return t

    def workspace(self, need, given, what):
        """``given``, or a fresh one of ``need`` bytes (0: the sizes are not served)."""
        if need == 0:
            raise HimuonError(-2, what + "_workspace_size")
        if given is None:
            given = self.empty(need, _torch().uint8)
        elif given.device != self.dev:
            raise ValueError("the workspace must be on the tensors' device")
        return given.data_ptr(), given.numel() * given.element_size()


def _done(status, what):
    if status != OK:
        raise HimuonError(status, what)


# -------------------------------------------------------------------- token table

def embed(tokens, table, scale=1.0, out=None, stream=None):
    """``scale * table[tokens]``: a tensor of ``tokens.shape + (width,)`` in the
    table's type. ``tokens`` is a contiguous int32 or int64 tensor; a token
    outside the table (such as -1 for padding) gives zeros. Rows of ``table`` and
    of a 2-D ``out`` (one row per token) may be strided."""
    _torch()
    ld = _matrix(table, "table")
    if not tokens.is_cuda or not tokens.is_contiguous():
        raise ValueError("tokens must be a contiguous CUDA tensor")
    dev, code, index = table.device, _dtype_code(table), _index_code(tokens)
    n, width = tokens.numel(), table.shape[1]
    with _Call(dev, stream) as call:
        if out is None:
            out = call.empty((*tokens.shape, width), table.dtype)
            ld_out = width
        else:
            if out.dtype != table.dtype or tuple(out.shape) not in ((n, width), (*tokens.shape, width)):
                raise ValueError("out must hold one row of the table's type and width per token")
            if out.dim() != 2 and not out.is_contiguous():
                raise ValueError("out must be a 2-D row-major or a contiguous tensor")
            ld_out = _matrix(out, "out") if out.dim() == 2 else width
        _same_device(dev, tokens, out)
        _done(lib().himuon_embed(n, tokens.data_ptr(), index, table.shape[0], width, table.data_ptr(), ld, out.data_ptr(),
                                 ld_out, float(scale), code, call.raw), "himuon_embed")
    return out


def embed_grad(tokens, grad, num_rows, scale=1.0, out=None, dtype=None, accumulate=False, workspace=None, stream=None):
    """The gradient of the table that ``embed`` read: row v of the result is
    ``scale`` times the sum of ``grad``'s rows whose token is v, summed in fp32 in
    an order that depends on the tokens alone. ``grad`` has one row per token
    (``tokens.shape + (width,)`` or 2-D with strided rows); the result is
    ``num_rows`` x width in ``dtype`` (default: ``grad``'s), or is added to ``out``
    with ``accumulate``."""
    torch = _torch()
    if not tokens.is_cuda or not tokens.is_contiguous():
        raise ValueError("tokens must be a contiguous CUDA tensor")
    n = tokens.numel()
    if grad.dim() != 2:
        if tuple(grad.shape[:-1]) != tuple(tokens.shape) or not grad.is_contiguous():
            raise ValueError("grad must have one row per token")
        grad = grad.view(n, grad.shape[-1])
    ld = _matrix(grad, "grad")
    if grad.shape[0] != n:
        raise ValueError("grad must have one row per token")
    dev, code, index, width, rows = grad.device, _dtype_code(grad), _index_code(tokens), grad.shape[1], int(num_rows)
    if accumulate and out is None:
        raise ValueError("accumulate needs the tensor to add to")
    with _Call(dev, stream) as call:
        if out is None:
            out = call.empty((rows, width), grad.dtype if dtype is None else dtype)
        elif tuple(out.shape) != (rows, width) or (dtype is not None and out.dtype != dtype):
            raise ValueError("out must be num_rows x width of the asked type")
        ld_out = _matrix(out, "out")
        _same_device(dev, tokens, out)
        L = lib()
        ws = call.workspace(L.himuon_embed_grad_workspace_size(n, rows, width), workspace, "himuon_embed_grad")
        _done(L.himuon_embed_grad(n, tokens.data_ptr(), index, rows, width, grad.data_ptr(), ld, code, out.data_ptr(), ld_out,
                                  _dtype_code(out), float(scale), int(bool(accumulate)), *ws, call.raw), "himuon_embed_grad")
    return out


# --------------------------------------------------------------- queries and keys

def _heads(t, what, like=None):
    """A [batch, seq, heads, dim] or [tokens, heads, dim] tensor as himuon_heads_t."""
    if t.dim() not in (3, 4) or not t.is_cuda or (t.stride(-1) != 1 and t.shape[-1] > 1):
        raise ValueError(f"{what} must be a [batch, seq, heads, dim] or [tokens, heads, dim] CUDA tensor with adjacent dim")
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{what} must match the inputs' shape, type and device")
    s = t.stride()
    return Heads(t.data_ptr(), s[0] if len(s) == 4 else 0, s[-3], s[-2])


def _qk_args(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved):
    torch = _torch()
    hq, hk = _heads(q, "q"), _heads(k, "k")
    if q.dim() != k.dim() or q.shape[:-2] != k.shape[:-2] or q.shape[-1] != k.shape[-1] or q.dtype != k.dtype:
        raise ValueError("q and k must share tokens, head size and type")
    dim = q.shape[-1]
    for g in (q_gain, k_gain):
        if tuple(g.shape) != (dim,) or g.dtype != q_gain.dtype or not g.is_contiguous():
            raise ValueError("gains must be contiguous tensors of the head size and of one type")
    if cos.dim() != 2 or cos.shape != sin.shape or cos.dtype != torch.float32 or sin.dtype != torch.float32 or \
            not cos.is_contiguous() or not sin.is_contiguous():
        raise ValueError("cos and sin must be contiguous float32 tensors, one row per position")
    _same_device(q.device, k, q_gain, k_gain, cos, sin, positions)
    index = I64
    if positions is not None:
        index = _index_code(positions)
        if positions.shape != q.shape[:-2] or not positions.is_contiguous():
            raise ValueError("positions must be a contiguous tensor, one per token")
    batch, seq = (q.shape[0], q.shape[1]) if q.dim() == 4 else (1, q.shape[0])
    return Qk(batch, seq, q.shape[-2], k.shape[-2], dim, 2 * cos.shape[1], int(bool(interleaved)), _dtype_code(q),
              _dtype_code(q_gain), index, q_gain.data_ptr(), k_gain.data_ptr(), cos.data_ptr(), sin.data_ptr(), cos.shape[0],
              positions.data_ptr() if positions is not None else None, float(eps)), hq, hk


def qk_norm_rope(q, k, q_gain, k_gain, cos, sin, positions=None, eps=1e-6, interleaved=False, out=None, stream=None):
    """Queries and keys, normalised per head, scaled by their gains and rotated by
    their positions, in one pass: (q', k').

    ``q``, ``k``      [batch, seq, heads, dim] or [tokens, heads, dim], any strides but
                    for adjacent elements of a head (slices of a fused projection).
    ``cos``, ``sin``  float32, row p the cosines and sines of position p's angles; twice
                    their width is the part of a head that is rotated.
    ``positions``   int32 or int64, one per token (default: the index in the
                    sequence). A position outside the table marks a token that is
                    not in use: zeros come out.
    ``interleaved`` pairs (2i, 2i+1) instead of (i, i + width).
    ``out``         the two tensors to write (q and k themselves are allowed)."""
    torch = _torch()
    args, hq, hk = _qk_args(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    with _Call(q.device, stream) as call:
        oq, ok = out if out is not None else (call.empty(q.shape, q.dtype), call.empty(k.shape, k.dtype))
        ref = ctypes.byref
        ho, hp = _heads(oq, "out", q), _heads(ok, "out", k)
        _done(lib().himuon_qk_norm_rope(ref(args), ref(hq), ref(hk), ref(ho), ref(hp), call.raw), "himuon_qk_norm_rope")
    return oq, ok


def qk_norm_rope_grad(g_q, g_k, q, k, q_gain, k_gain, cos, sin, positions=None, eps=1e-6, interleaved=False, out=None,
                      workspace=None, stream=None):
    """The backward pass of ``qk_norm_rope``: from the gradients ``g_q``, ``g_k`` of its
    outputs and its inputs, (dq, dk, dq_gain, dk_gain). ``out``: the tensors for dq
    and dk (``g_q`` and ``g_k`` themselves are allowed)."""
    torch = _torch()
    args, hq, hk = _qk_args(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    gq, gk = _heads(g_q, "g_q", q), _heads(g_k, "g_k", k)
    with _Call(q.device, stream) as call:
        oq, ok = out if out is not None else (call.empty(q.shape, q.dtype), call.empty(k.shape, k.dtype))
        dwq, dwk = (call.empty(w.shape, w.dtype) for w in (q_gain, k_gain))
        ref = ctypes.byref
        ho, hp = _heads(oq, "out", q), _heads(ok, "out", k)
        L = lib()
        ws = call.workspace(L.himuon_qk_norm_rope_grad_workspace_size(args.batch, args.seq, args.head_dim), workspace,
                            "himuon_qk_norm_rope_grad")
        _done(L.himuon_qk_norm_rope_grad(ref(args), ref(gq), ref(gk), ref(hq), ref(hk), ref(ho), ref(hp), dwq.data_ptr(),
                                         dwk.data_ptr(), *ws, call.raw), "himuon_qk_norm_rope_grad")
    return oq, ok, dwq, dwk


# ------------------------------------------------------------- activations in 8 bits

def _packed(codes, exps):
    """Checks an activation in 8 bits; (groups, columns)."""
    torch = _torch()
    if codes.dtype != torch.uint8 or exps.dtype != torch.uint8 or codes.dim() != 3 or codes.shape[2] != ACT_GROUP or \
            codes.shape[:2] != exps.shape or not codes.is_contiguous() or not exps.is_contiguous() or not codes.is_cuda:
        raise ValueError("codes must be a contiguous uint8 CUDA tensor [groups, columns, 32], exponents [groups, columns]")
    _same_device(codes.device, exps)
    return exps.shape


def act_pack(x, out=None, stream=None):
    """A [tokens, columns] activation in 8 bits: (codes, exponents), uint8 tensors of
    shapes [ceil(tokens / 32), columns, 32] and [ceil(tokens / 32), columns]. 32
    tokens of a column share a power of two; a value keeps four significant bits."""
    torch = _torch()
    ld = _matrix(x, "x")
    n, cols = x.shape
    shape = (-(-n // ACT_GROUP), cols)
    with _Call(x.device, stream) as call:
        codes, exps = out if out is not None else (call.empty((*shape, ACT_GROUP), torch.uint8), call.empty(shape, torch.uint8))
        if tuple(_packed(codes, exps)) != shape:
            raise ValueError("out must be codes [ceil(tokens / 32), columns, 32] and exponents [ceil(tokens / 32), columns]")
        _same_device(x.device, codes)
        _done(lib().himuon_act_pack(n, cols, x.data_ptr(), ld, _dtype_code(x), codes.data_ptr(), exps.data_ptr(), call.raw),
              "himuon_act_pack")
    return codes, exps


def act_unpack(codes, exps, tokens, dtype=None, out=None, stream=None):
    """The [tokens, columns] values that ``act_pack``'s result stands for, in
    ``dtype`` (bfloat16 by default; exact in both types)."""
    torch = _torch()
    groups, cols = _packed(codes, exps)
    n = int(tokens)
    if n < 0 or -(-n // ACT_GROUP) != groups:
        raise ValueError("tokens does not match the number of groups")
    with _Call(codes.device, stream) as call:
        if out is None:
            out = call.empty((n, cols), torch.bfloat16 if dtype is None else dtype)
        elif tuple(out.shape) != (n, cols) or (dtype is not None and out.dtype != dtype):
            raise ValueError("out must be tokens x columns of the asked type")
        ld = _matrix(out, "out")
        _same_device(codes.device, out)
        _done(lib().himuon_act_unpack(n, cols, codes.data_ptr(), exps.data_ptr(), out.data_ptr(), ld, _dtype_code(out), call.raw),
              "himuon_act_unpack")
    return out


def weight_grad(grad, codes, exps, out=None, dtype=None, accumulate=False, workspace=None, stream=None):
    """The gradient of a weight matrix, ``grad.T @ x``, from the gradient of its
    outputs [tokens, rows] and its inputs x held in 8 bits: rows x columns in
    ``dtype`` (default: ``grad``'s), or added to ``out`` with ``accumulate``. The result
    may be what ``step`` takes as a gradient."""
    _torch()
    ld = _matrix(grad, "grad")
    groups, cols = _packed(codes, exps)
    n, rows = grad.shape
    if -(-n // ACT_GROUP) != groups:
        raise ValueError("grad and the activation differ in tokens")
    if accumulate and out is None:
        raise ValueError("accumulate needs the tensor to add to")
    code = _dtype_code(grad)
    with _Call(grad.device, stream) as call:
        if out is None:
            out = call.empty((rows, cols), grad.dtype if dtype is None else dtype)
        elif tuple(out.shape) != (rows, cols) or (dtype is not None and out.dtype != dtype):
            raise ValueError("out must be rows x columns of the asked type")
        ld_out = _matrix(out, "out")
        _same_device(grad.device, codes, out)
        L = lib()
        ws = call.workspace(L.himuon_weight_grad_workspace_size(n, rows, cols, grad.data_ptr(), ld, code), workspace, "himuon_weight_grad")
        _done(L.himuon_weight_grad(n, rows, cols, grad.data_ptr(), ld, code, codes.data_ptr(), exps.data_ptr(), out.data_ptr(),
                                   ld_out, _dtype_code(out), int(bool(accumulate)), *ws, call.raw), "himuon_weight_grad")
    return out
