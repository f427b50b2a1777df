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

``embed`` and ``qk_norm_rope`` join autograd where it records: gradients reach the table,
queries, keys and gains (not the cosines and sines). Results written to ``out``, and the
other operators' results, carry no graph. Neither has a forward-mode derivative: tensors with
tangents are refused, by their gradients too, and so are scales and eps that are tensors
which ask for a gradient.

Inputs of a call for another stream are the caller's to keep until it has read them
(``record_stream``), as with torch's own operations.
"""
from __future__ import annotations

import ctypes
import struct

from . import BF16, F32, OK, HimuonError, _dtype_code, lib

I32, I64 = 0, 1              # himuon_index_t
MAX_HEAD_DIM = 512           # HIMUON_MAX_HEAD_DIM
ACT_GROUP = 32               # HIMUON_ACT_GROUP: tokens of a column that share an exponent

_i64, _vp, _sz, _f, _int = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float, ctypes.c_int


# himuon_heads_t and himuon_qk_t, as bytes (a call packs them in one go)
_HEADS = struct.Struct("@P3q")
_QK = struct.Struct("@2q8i4PqPf0q")


def declare(L):
    """Argument types of the operators' entry points (called once, as the library is loaded)."""
    L.himuon_embed.argtypes = [_i64, _vp, _int, _i64, _i64, _vp, _i64, _vp, _i64, _f, _int, _vp]
    L.himuon_embed_grad_workspace_size.argtypes = [_i64, _i64, _i64]
    L.himuon_embed_grad.argtypes = [_i64, _vp, _int, _i64, _i64, _vp, _i64, _int, _vp, _i64, _int, _f, _int, _vp, _sz, _vp]
    L.himuon_qk_norm_rope.argtypes = [_vp] * 6
    L.himuon_qk_norm_rope_grad_workspace_size.argtypes = [_i64, _i64, _i64]
    L.himuon_qk_norm_rope_grad.argtypes = [_vp] * 10 + [_sz, _vp]
    L.himuon_act_pack.argtypes = [_i64, _i64, _vp, _i64, _int, _vp, _vp, _vp]
    L.himuon_act_unpack.argtypes = [_i64, _i64, _vp, _vp, _vp, _i64, _int, _vp]
    L.himuon_weight_grad_workspace_size.argtypes = [_i64, _i64, _i64, _vp, _i64, _int]
    L.himuon_weight_grad.argtypes = [_i64, _i64, _i64, _vp, _i64, _int, _vp, _vp, _vp, _i64, _int, _int, _vp, _sz, _vp]
    for name in ("embed", "embed_grad", "qk_norm_rope", "qk_norm_rope_grad", "act_pack", "act_unpack", "weight_grad"):
        getattr(L, "himuon_" + name).restype = _int
    for name in ("embed_grad", "qk_norm_rope_grad", "weight_grad"):
        getattr(L, f"himuon_{name}_workspace_size").restype = _sz


# ------------------------------------------------------------------ shared checks
#
# (These run on every call: a small call's time is the host's. Tensors' properties are read
# once, and the error messages are made only when something is wrong.)

_INDEX, _TYPES = {}, {}
_device = _raw_stream = _forward = None


def _torch():
    global _device, _raw_stream, _forward
    import torch
    if not _INDEX:  # (filled last: another thread that finds it filled finds all of this)
        _device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        from torch.autograd import forward_ad as _forward
        _TYPES.update({torch.float32: F32, torch.bfloat16: BF16})
        _INDEX.update({torch.int32: I32, torch.int64: I64})
    return torch


def _index_code(t):
    code = _INDEX.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported index type {t.dtype}; expected int32 or int64")
    return code


def _type_code(t):
    code = _TYPES.get(t.dtype)
    return _dtype_code(t) if code is None else code


def _keeps(op, number, *tensors):
    """Refuses what would lose a derivative without a word: a tensor with a tangent (the operators
    have no forward-mode rules), and a number that is a tensor which asks for a gradient."""
    if _forward is not None and _forward._current_level < 0 and (type(number) is float or number is None):
        return
    torch = _torch()
    if getattr(number, "requires_grad", False) and torch.is_grad_enabled():
        raise NotImplementedError(f"{op} gives no gradient of its scale or eps: pass a number, or the tensor detached")
    if _forward._current_level >= 0:
        for t in (number, *tensors):
            if isinstance(t, torch.Tensor) and _forward.unpack_dual(t).tangent is not None:
                raise NotImplementedError(f"{op} has no forward-mode derivative: its arguments must not carry tangents")


def _matrix(t, what):
    """Checks a row-major CUDA matrix; (rows, columns, leading dimension)."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or not t.is_cuda or (stride[1] != 1 and shape[1] > 1):
        raise ValueError(f"{what} must be a 2-D row-major CUDA tensor")
    rows, cols = shape
    return rows, cols, (stride[0] if rows > 1 else max(cols, 1))


def _same_device(dev, *tensors):
    for t in tensors:
        if t is not None and t.device != dev:
            raise ValueError("tensors must be on one device")


def _away(dev, stream):
    """Whether a call is for another device or stream than the current ones."""
    index = dev.index
    return index != _device() or (stream is not None and (stream.cuda_stream != _raw_stream(index) or stream.device != dev))


def _on(dev, stream, f, *args):
    """``f(*args)`` with ``dev`` the current device (the default stream has no handle that
    names its device) and ``stream`` the current stream: what the call allocates is then
    that stream's memory, of which no work on another stream is left. Results may be read
    and freed on the stream that was current before."""
    torch = _torch()
    if stream is None:
        with torch.cuda.device(dev):
            return f(*args)
    if stream.device != dev:
        raise ValueError("the stream must be on the tensors' device")
    here = torch.cuda.current_stream(dev)
    with torch.cuda.stream(stream):
        result = f(*args)
    if stream != here:
        for t in result if isinstance(result, tuple) else (result,):
            t.record_stream(here)
    return result


def _stream_of(index):
    return _raw_stream(index) or None


def _new(like, shape, dtype):
    """A fresh tensor on ``like``'s device, of its type unless another one is asked for."""
    if dtype is None or dtype == like.dtype:
        return like.new_empty(shape)
    return _torch().empty(shape, dtype=dtype, device=like.device)


def _workspace(need, given, like):
    """(tensor, address, bytes) of ``given``, or of a fresh workspace of ``need`` bytes (none
    for 0: the call needs none, or reports what is wrong with it). The caller holds the
    tensor until its work is enqueued."""
    if given is None:
        if need == 0:
            return None, None, 0
        torch = _torch()
        given = torch.empty(need, dtype=torch.uint8, device=like.device)
        return given, given.data_ptr(), need
    if given.device != like.device or not given.is_contiguous():  # (its bytes are counted by its elements)
        raise ValueError("the workspace must be a contiguous tensor on the tensors' device")
    return given, given.data_ptr(), given.numel() * given.element_size()


def _functions():
    from . import train_autograd  # (torch itself is imported by the first call)
    return train_autograd


def _done(status, what):
    if status != OK:
        raise HimuonError(status, what)


# -------------------------------------------------------------------- token table

def embed(tokens, table, scale=1.0, out=None, stream=None):
    """``scale * table[tokens]``: a tensor of ``tokens.shape + (width,)`` in the
    table's type. ``tokens`` is a contiguous int32 or int64 tensor; a token
    outside the table (such as -1 for padding) gives zeros. Rows of ``table`` and
    of a 2-D ``out`` (one row per token) may be strided. The table's gradient is
    ``embed_grad``'s."""
    torch = _torch()
    _keeps("embed", scale, table)
    rows, width, ld = _matrix(table, "table")
    if not tokens.is_cuda or not tokens.is_contiguous():
        raise ValueError("tokens must be a contiguous CUDA tensor")
    dev, n = table.device, tokens.numel()
    if _away(dev, stream):
        return _on(dev, stream, embed, tokens, table, scale, out)
    if table.requires_grad and out is None and torch.is_grad_enabled():
        return _functions().Embed.apply(tokens, table, scale)
    code, index = _type_code(table), _index_code(tokens)
    if out is None:
        out = table.new_empty((*tokens.shape, width))
        ld_out = width
        _same_device(dev, tokens)
    else:
        if out.dtype != table.dtype or tuple(out.shape) not in ((n, width), (*tokens.shape, width)):
            raise ValueError("out must hold one row of the table's type and width per token")
        if out.dim() != 2 and not out.is_contiguous():
            raise ValueError("out must be a 2-D row-major or a contiguous tensor")
        ld_out = _matrix(out, "out")[2] if out.dim() == 2 else width
        _same_device(dev, tokens, out)
    _done(lib().himuon_embed(n, tokens.data_ptr(), index, rows, width, table.data_ptr(), ld, out.data_ptr(), ld_out,
                             scale, code, _stream_of(dev.index)), "himuon_embed")
    return out


def embed_grad(tokens, grad, num_rows, scale=1.0, out=None, dtype=None, accumulate=False, workspace=None, stream=None):
    """The gradient of the table that ``embed`` read: row v of the result is
    ``scale`` times the sum of ``grad``'s rows whose token is v, summed in fp32 in
    an order that depends on the tokens alone. ``grad`` has one row per token
    (``tokens.shape + (width,)`` or 2-D with strided rows); the result is
    ``num_rows`` x width in ``dtype`` (default: ``grad``'s), or is added to ``out``
    with ``accumulate``."""
    _keeps("embed_grad", scale, grad, out)
    if not tokens.is_cuda or not tokens.is_contiguous():
        raise ValueError("tokens must be a contiguous CUDA tensor")
    n = tokens.numel()
    if grad.dim() != 2:
        if tuple(grad.shape[:-1]) != tuple(tokens.shape) or not grad.is_contiguous():
            raise ValueError("grad must have one row per token")
        grad = grad.view(n, grad.shape[-1])
    given, width, ld = _matrix(grad, "grad")
    if given != n:
        raise ValueError("grad must have one row per token")
    if accumulate and out is None:
        raise ValueError("accumulate needs the tensor to add to")
    dev, rows = grad.device, int(num_rows)
    if _away(dev, stream):
        return _on(dev, stream, embed_grad, tokens, grad, rows, scale, out, dtype, accumulate, workspace)
    code, index = _type_code(grad), _index_code(tokens)
    L = lib()
    held, ws, ws_bytes = _workspace(L.himuon_embed_grad_workspace_size(n, rows, width), workspace, grad)
    if out is None:
        out = _new(grad, (rows, width), dtype)
    elif tuple(out.shape) != (rows, width) or (dtype is not None and out.dtype != dtype):
        raise ValueError("out must be num_rows x width of the asked type")
    ld_out = _matrix(out, "out")[2]
    _same_device(dev, tokens, out)
    _done(L.himuon_embed_grad(n, tokens.data_ptr(), index, rows, width, grad.data_ptr(), ld, code, out.data_ptr(), ld_out,
                              _type_code(out), scale, bool(accumulate), ws, ws_bytes, _stream_of(dev.index)),
          "himuon_embed_grad")
    return out


# --------------------------------------------------------------- queries and keys

def _heads(t, what):
    """A [batch, seq, heads, dim] or [tokens, heads, dim] tensor: its shape, and himuon_heads_t."""
    shape, s = tuple(t.shape), t.stride()
    n = len(shape)
    if n == 4:
        packed = _HEADS.pack(t.data_ptr(), s[0], s[1], s[2])
    elif n == 3:
        packed = _HEADS.pack(t.data_ptr(), 0, s[0], s[1])
    else:
        n = 0
    if n == 0 or not t.is_cuda or (s[-1] != 1 and shape[-1] > 1):
        raise ValueError(f"{what} must be a [batch, seq, heads, dim] or [tokens, heads, dim] CUDA tensor with adjacent dim")
    return shape, packed


def _heads_like(t, what, shape, like):
    got, packed = _heads(t, what)
    if got != shape or t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{what} must match the inputs' shape, type and device")
    return packed


def _outputs(out, q, k, sq, sk):
    """The two output tensors (fresh ones if ``out`` is None), and both as himuon_heads_t."""
    if out is not None:
        oq, ok = out
        return oq, ok, _heads_like(oq, "out", sq, q), _heads_like(ok, "out", sk, k)
    oq, ok = q.new_empty(sq), k.new_empty(sk)
    seq, hq, hk, dim = sq[-3], sq[-2], sk[-2], sq[-1]
    return (oq, ok, _HEADS.pack(oq.data_ptr(), seq * hq * dim, hq * dim, dim),
            _HEADS.pack(ok.data_ptr(), seq * hk * dim, hk * dim, dim))


def _qk_args(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved):
    """(shape of q, of k, himuon_qk_t, and q and k as himuon_heads_t), checked."""
    torch = _torch()
    sq, hq = _heads(q, "q")
    sk, hk = _heads(k, "k")
    dim, dev, f32 = sq[-1], q.device, torch.float32
    if sq[:-2] != sk[:-2] or dim != sk[-1] or q.dtype != k.dtype:
        raise ValueError("q and k must share tokens, head size and type")
    gain = q_gain.dtype
    if q_gain.shape != (dim,) or k_gain.shape != (dim,) or k_gain.dtype != gain or not q_gain.is_contiguous() or \
            not k_gain.is_contiguous():
        raise ValueError("gains must be contiguous tensors of the head size and of one type")
    table = cos.shape
    if len(table) != 2 or sin.shape != table or cos.dtype != f32 or sin.dtype != f32 or not cos.is_contiguous() or \
            not sin.is_contiguous():
        raise ValueError("cos and sin must be contiguous float32 tensors, one row per position")
    _same_device(dev, k, q_gain, k_gain, cos, sin, positions)
    index, at = I64, 0
    if positions is not None:
        index, at = _index_code(positions), positions.data_ptr()
        if tuple(positions.shape) != sq[:-2] or not positions.is_contiguous():
            raise ValueError("positions must be a contiguous tensor, one per token")
    batch, seq = (sq[0], sq[1]) if len(sq) == 4 else (1, sq[0])
    return sq, sk, _QK.pack(batch, seq, sq[-2], sk[-2], dim, 2 * table[1], bool(interleaved), _type_code(q), _type_code(q_gain),
                            index, q_gain.data_ptr(), k_gain.data_ptr(), cos.data_ptr(), sin.data_ptr(), table[0], at, eps), hq, hk


def qk_norm_rope(q, k, q_gain, k_gain, cos, sin, positions=None, eps=1e-6, interleaved=False, out=None, stream=None):
    """Queries and keys, normalised per head, scaled by their gains and rotated by
    their positions, in one pass: (q', k').

    ``q``, ``k``      [batch, seq, heads, dim] or [tokens, heads, dim], any strides but
                    for adjacent elements of a head (slices of a fused projection).
    ``cos``, ``sin``  float32, row p the cosines and sines of position p's angles; twice
                    their width is the part of a head that is rotated.
    ``positions``   contiguous int32 or int64, one per token (default: the index in the
                    sequence). A position outside the table marks a token that is
                    not in use: zeros come out.
    ``interleaved`` pairs (2i, 2i+1) instead of (i, i + width).
    ``out``         the two tensors to write (q and k themselves are allowed).

    The gradients of ``q``, ``k`` and the gains are ``qk_norm_rope_grad``'s."""
    _keeps("qk_norm_rope", eps, q, k, q_gain, k_gain, cos, sin)
    sq, sk, args, hq, hk = _qk_args(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    dev = q.device
    if _away(dev, stream):
        return _on(dev, stream, qk_norm_rope, q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, out)
    if out is None and (q.requires_grad or k.requires_grad or q_gain.requires_grad or k_gain.requires_grad) and \
            _torch().is_grad_enabled():
        return _functions().QkNormRope.apply(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    oq, ok, ho, hp = _outputs(out, q, k, sq, sk)
    _done(lib().himuon_qk_norm_rope(args, hq, hk, ho, hp, _stream_of(dev.index)), "himuon_qk_norm_rope")
    return oq, ok


def qk_norm_rope_grad(g_q, g_k, q, k, q_gain, k_gain, cos, sin, positions=None, eps=1e-6, interleaved=False, out=None,
                      workspace=None, stream=None):
    """The backward pass of ``qk_norm_rope``: from the gradients ``g_q``, ``g_k`` of its
    outputs and its inputs, (dq, dk, dq_gain, dk_gain). ``out``: the tensors for dq
    and dk (``g_q`` and ``g_k`` themselves are allowed)."""
    torch = _torch()
    _keeps("qk_norm_rope_grad", eps, g_q, g_k, q, k, q_gain, k_gain, cos, sin)
    sq, sk, args, hq, hk = _qk_args(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    dev = q.device
    if _away(dev, stream):
        return _on(dev, stream, qk_norm_rope_grad, g_q, g_k, q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, out,
                   workspace)
    gq, gk = _heads_like(g_q, "g_q", sq, q), _heads_like(g_k, "g_k", sk, k)
    L = lib()
    batch, seq = (sq[0], sq[1]) if len(sq) == 4 else (1, sq[0])
    held, ws, ws_bytes = _workspace(L.himuon_qk_norm_rope_grad_workspace_size(batch, seq, sq[-1]), workspace, q)
    oq, ok, ho, hp = _outputs(out, q, k, sq, sk)
    dwq, dwk = torch.empty_like(q_gain), torch.empty_like(k_gain)
    _done(L.himuon_qk_norm_rope_grad(args, gq, gk, hq, hk, ho, hp, dwq.data_ptr(), dwk.data_ptr(), ws, ws_bytes,
                                     _stream_of(dev.index)),
          "himuon_qk_norm_rope_grad")
    return oq, ok, dwq, dwk


# ------------------------------------------------------------- activations in 8 bits

def _packed(codes, exps):
    """Checks an activation in 8 bits; (groups, columns)."""
    u8, shape = _torch().uint8, codes.shape
    if codes.dtype != u8 or exps.dtype != u8 or len(shape) != 3 or shape[2] != ACT_GROUP or shape[:2] != exps.shape or \
            not codes.is_contiguous() or not exps.is_contiguous() or not codes.is_cuda:
        raise ValueError("codes must be a contiguous uint8 CUDA tensor [groups, columns, 32], exponents [groups, columns]")
    _same_device(codes.device, exps)
    return shape[0], shape[1]


def act_pack(x, out=None, stream=None):
    """A [tokens, columns] activation in 8 bits: (codes, exponents), uint8 tensors of
    shapes [ceil(tokens / 32), columns, 32] and [ceil(tokens / 32), columns]. 32
    tokens of a column share a power of two; a value keeps four significant bits."""
    torch = _torch()
    n, cols, ld = _matrix(x, "x")
    dev, code, groups = x.device, _type_code(x), -(-n // ACT_GROUP)
    if _away(dev, stream):
        return _on(dev, stream, act_pack, x, out)
    if out is None:
        codes = torch.empty((groups, cols, ACT_GROUP), dtype=torch.uint8, device=dev)
        exps = codes.new_empty((groups, cols))
    else:
        codes, exps = out
        if _packed(codes, exps) != (groups, cols):
            raise ValueError("out must be codes [ceil(tokens / 32), columns, 32] and exponents [ceil(tokens / 32), columns]")
        _same_device(dev, codes)
    _done(lib().himuon_act_pack(n, cols, x.data_ptr(), ld, code, codes.data_ptr(), exps.data_ptr(),
                                _stream_of(dev.index)), "himuon_act_pack")
    return codes, exps


def act_unpack(codes, exps, tokens, dtype=None, out=None, stream=None):
    """The [tokens, columns] values that ``act_pack``'s result stands for, in
    ``dtype`` (bfloat16 by default; exact in both types)."""
    torch = _torch()
    groups, cols = _packed(codes, exps)
    n, dev = int(tokens), codes.device
    if n < 0 or -(-n // ACT_GROUP) != groups:
        raise ValueError("tokens does not match the number of groups")
    if _away(dev, stream):
        return _on(dev, stream, act_unpack, codes, exps, n, dtype, out)
    if out is None:
        out = torch.empty((n, cols), dtype=torch.bfloat16 if dtype is None else dtype, device=dev)
    elif tuple(out.shape) != (n, cols) or (dtype is not None and out.dtype != dtype):
        raise ValueError("out must be tokens x columns of the asked type")
    ld = _matrix(out, "out")[2]
    _same_device(dev, out)
    _done(lib().himuon_act_unpack(n, cols, codes.data_ptr(), exps.data_ptr(), out.data_ptr(), ld, _type_code(out),
                                  _stream_of(dev.index)), "himuon_act_unpack")
    return out


def weight_grad(grad, codes, exps, out=None, dtype=None, accumulate=False, workspace=None, stream=None):
    """The gradient of a weight matrix, ``grad.T @ x``, from the gradient of its
    outputs [tokens, rows] and its inputs x held in 8 bits: rows x columns in
    ``dtype`` (default: ``grad``'s), or added to ``out`` with ``accumulate``. The result
    may be what ``step`` takes as a gradient."""
    _torch()
    n, rows, ld = _matrix(grad, "grad")
    groups, cols = _packed(codes, exps)
    if -(-n // ACT_GROUP) != groups:
        raise ValueError("grad and the activation differ in tokens")
    if accumulate and out is None:
        raise ValueError("accumulate needs the tensor to add to")
    code, dev, at = _type_code(grad), grad.device, grad.data_ptr()
    if _away(dev, stream):
        return _on(dev, stream, weight_grad, grad, codes, exps, out, dtype, accumulate, workspace)
    L = lib()
    held, ws, ws_bytes = _workspace(L.himuon_weight_grad_workspace_size(n, rows, cols, at, ld, code), workspace, grad)
    if out is None:
        out = _new(grad, (rows, cols), dtype)
    elif tuple(out.shape) != (rows, cols) or (dtype is not None and out.dtype != dtype):
        raise ValueError("out must be rows x columns of the asked type")
    ld_out = _matrix(out, "out")[2]
    _same_device(dev, codes, out)
    _done(L.himuon_weight_grad(n, rows, cols, at, ld, code, codes.data_ptr(), exps.data_ptr(), out.data_ptr(), ld_out,
                               _type_code(out), bool(accumulate), ws, ws_bytes, _stream_of(dev.index)),
          "himuon_weight_grad")
    return out
