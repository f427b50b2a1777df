"""The operators of a decoder block's training step between its projections, on tensors.

``add_norm`` / ``add_norm_grad``              the residual's addition and the norm of the sum,
                                            in 8 bits too on request
``attention`` / ``attention_grad``            attention with grouped heads over whole sequences
``token_logprob`` / ``token_logprob_grad``    log probabilities of given tokens, entropies and
                                            the most likely tokens: the loss

They keep the rules of ``train_ops``: argument checks and marshalling only, work on
``stream`` (default: torch's current stream), fresh results unless ``out`` is given,
HimuonError for an error of the library; float32 or bfloat16 storage.

``add_norm``, ``attention`` and ``token_logprob`` join autograd where it records (results
written to ``out`` carry no graph). lse and the most likely tokens carry none. Tensors with
tangents are refused (there are no forward-mode derivatives), and so are scales and eps that are
tensors which ask for a gradient. A backward
pass is captured into a HIP graph as any of torch's is: after a warm-up on the capturing
stream, and while no eager graph of the same leaves is alive.
"""
from __future__ import annotations

import ctypes
import struct

from . import lib
from .train_ops import (ACT_GROUP, I32, _away, _done, _heads, _heads_like, _HEADS, _index_code, _keeps, _matrix, _on, _same_device,
                        _stream_of, _torch, _type_code, _workspace)

MAX_ATTN_DIM = 256           # HIMUON_MAX_ATTN_DIM
MAX_TOP = 64                 # HIMUON_MAX_TOP

_i64, _vp, _sz, _f, _int = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float, ctypes.c_int

_ATTN = struct.Struct("@3q6i4Pf0q")  # himuon_attn_t


def declare(L):
    """Argument types of the operators' entry points (called once, as the library is loaded)."""
    L.himuon_add_norm.argtypes = [_i64, _i64, _vp, _i64, _vp, _i64, _vp, _int, _vp, _i64, _vp, _i64, _vp, _vp, _f, _int, _vp]
    L.himuon_add_norm_grad_workspace_size.argtypes = [_i64, _i64]
    L.himuon_add_norm_grad.argtypes = [_i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _int, _vp, _i64, _vp, _f, _int, _vp, _sz,
                                       _vp]
    L.himuon_attention_workspace_size.argtypes = [_vp]
    L.himuon_attention.argtypes = [_vp] * 7 + [_sz, _vp]
    L.himuon_attention_grad_workspace_size.argtypes = [_vp]
    L.himuon_attention_grad.argtypes = [_vp] * 11 + [_sz, _vp]
    L.himuon_token_logprob.argtypes = [_i64, _i64, _vp, _i64, _int, _vp, _int, _f, _int, _vp, _vp, _vp, _vp, _vp, _vp]
    L.himuon_token_logprob_grad.argtypes = [_i64, _i64, _vp, _vp, _vp, _i64, _int, _vp, _int, _vp, _vp, _f, _vp, _i64, _vp]
    for name in ("add_norm", "add_norm_grad", "attention", "attention_grad", "token_logprob", "token_logprob_grad"):
        getattr(L, "himuon_" + name).restype = _int
    for name in ("add_norm_grad", "attention", "attention_grad"):
        getattr(L, f"himuon_{name}_workspace_size").restype = _sz


def _functions():
    from . import block_autograd  # (torch itself is imported by the first call)
    return block_autograd


# ----------------------------------------------------------------- residual and norm

def _rows(t, what):
    """(tokens, width, leading dimension) of a [..., width] tensor: contiguous, or 2-D with strided rows."""
    shape = t.shape
    if len(shape) == 2:
        return _matrix(t, what)
    if len(shape) < 2 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what} must be a 2-D row-major or a contiguous CUDA tensor [..., width]")
    width = shape[-1]
    return (t.numel() // width if width else 0), width, max(width, 1)


def _rows_like(t, what, like):
    if t.shape != like.shape or t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{what} must match the input's shape, type and device")
    return _rows(t, what)[2]


def _gain(gain, width):
    if gain.shape != (width,) or not gain.is_contiguous():
        raise ValueError("gain must be a contiguous tensor of the width")
    return _type_code(gain)


def add_norm(x, residual, gain, eps=1e-6, pack=False, out=None, stream=None):
    """``h = x + residual`` and ``y = h * gain / sqrt(mean(h * h) + eps)`` over the last
    dimension: (h, y), or with ``pack`` (h, y, codes, exponents), the last two what
    ``act_pack`` makes of y's rows, for ``weight_grad``. Without a residual (None) h is x itself.

    ``x``, ``residual``  [..., width], contiguous or 2-D with strided rows.
    ``gain``             [width], float32 or bfloat16.
    ``out``              the tensors (h, y) to write; h may be x or residual. (None, y)
                       where there is no residual.

    The gradients of ``x``, ``residual`` and ``gain`` are ``add_norm_grad``'s."""
    torch = _torch()
    _keeps("add_norm", eps, x, residual, gain)
    rows, width, ld = _rows(x, "x")
    dev, code, gain_code = x.device, _type_code(x), _gain(gain, width)
    ld_res = 0 if residual is None else _rows_like(residual, "residual", x)
    _same_device(dev, gain)
    if _away(dev, stream):
        return _on(dev, stream, add_norm, x, residual, gain, eps, pack, out)
    if out is None and (x.requires_grad or gain.requires_grad or (residual is not None and residual.requires_grad)) and \
            torch.is_grad_enabled():
        return _functions().AddNorm.apply(x, residual, gain, eps, pack) if residual is not None else \
            (x, *_functions().Norm.apply(x, gain, eps, pack))
    if out is None:
        h, y = None if residual is None else x.new_empty(x.shape), x.new_empty(x.shape)
        ld_h = ld_y = width
    else:
        h, y = out
        ld_y = _rows_like(y, "out", x)
        if (h is None) != (residual is None):
            raise ValueError("out holds h exactly where there is a residual")
        ld_h = 0 if h is None else _rows_like(h, "out", x)
    codes = exps = None
    if pack:
        groups = -(-rows // ACT_GROUP)
        codes = torch.empty((groups, width, ACT_GROUP), dtype=torch.uint8, device=dev)
        exps = codes.new_empty((groups, width))
    _done(lib().himuon_add_norm(rows, width, x.data_ptr(), ld, None if residual is None else residual.data_ptr(), ld_res,
                                gain.data_ptr(), gain_code, None if h is None else h.data_ptr(), ld_h, y.data_ptr(), ld_y,
                                codes.data_ptr() if pack else None, exps.data_ptr() if pack else None, eps, code,
                                _stream_of(dev.index)), "himuon_add_norm")
    h = x if h is None else h
    return (h, y, codes, exps) if pack else (h, y)


def add_norm_grad(g_y, h, gain, g_h=None, eps=1e-6, out=None, workspace=None, stream=None):
    """The backward pass of ``add_norm``: from the gradients ``g_y`` of y and ``g_h`` of h
    (None: h was not used further) and from h, (dh, dgain). dh is the gradient of x and of
    the residual alike. ``out``: the tensor for dh (``g_y`` or ``g_h`` is allowed)."""
    torch = _torch()
    _keeps("add_norm_grad", eps, g_y, h, gain, g_h)
    rows, width, ld = _rows(h, "h")
    dev, code, gain_code = h.device, _type_code(h), _gain(gain, width)
    ld_gy = _rows_like(g_y, "g_y", h)
    ld_gh = 0 if g_h is None else _rows_like(g_h, "g_h", h)
    _same_device(dev, gain)
    if _away(dev, stream):
        return _on(dev, stream, add_norm_grad, g_y, h, gain, g_h, eps, out, workspace)
    L = lib()
    held, ws, ws_bytes = _workspace(L.himuon_add_norm_grad_workspace_size(rows, width), workspace, h)
    if out is None:
        out, ld_out = h.new_empty(h.shape), width
    else:
        ld_out = _rows_like(out, "out", h)
    dgain = torch.empty_like(gain)
    _done(L.himuon_add_norm_grad(rows, width, g_y.data_ptr(), ld_gy, None if g_h is None else g_h.data_ptr(), ld_gh, h.data_ptr(), ld,
                                 gain.data_ptr(), gain_code, out.data_ptr(), ld_out, dgain.data_ptr(), eps, code, ws, ws_bytes,
                                 _stream_of(dev.index)), "himuon_add_norm_grad")
    return out, dgain


# ------------------------------------------------------------------------ attention

def _where(t, what, count, dev, index):
    """(address, index type) of an array of starts or lengths."""
    if t is None:
        return 0, index
    if tuple(t.shape) != (count,) or not t.is_contiguous() or t.device != dev:
        raise ValueError(f"{what} must be a contiguous tensor of {count} on the inputs' device")
    code = _index_code(t)
    if index is not None and code != index:
        raise ValueError("starts and lengths must be of one type")
    return t.data_ptr(), code


def _attn_args(q, k, v, q_starts, k_starts, q_lengths, k_lengths, causal, scale):
    """(shapes of q and k, himuon_attn_t, q, k and v as himuon_heads_t), checked."""
    sq, hq = _heads(q, "q")
    sk, hk = _heads(k, "k")
    dim, dev = sq[-1], q.device
    if len(sk) != len(sq) or sk[-1] != dim or k.dtype != q.dtype or k.device != dev:
        raise ValueError("q and k must share dimensions, head size, type and device")
    if dim < 1:
        raise ValueError("heads must have at least one element")
    hv = _heads_like(v, "v", sk, k)
    if sk[-2] < 1 or sq[-2] % sk[-2]:
        raise ValueError("the number of query heads must be a multiple of the number of key heads")
    if len(sq) == 4:
        if q_starts is not None or k_starts is not None:
            raise ValueError("starts are for packed sequences ([tokens, heads, dim])")
        if sk[0] != sq[0]:
            raise ValueError("q and k must share the batch")
        batch, n_q, n_k = sq[0], sq[1], sk[1]
        qs = ks = 0
        index = None
    else:
        n_q, n_k = sq[0], sk[0]
        if q_starts is None:
            if k_starts is not None:
                raise ValueError("k_starts without q_starts")
            batch, qs, ks, index = 1, 0, 0, None
        else:
            if k_starts is None:
                if n_q != n_k:
                    raise ValueError("k_starts may be left out only where q and k have the same tokens")
                k_starts = q_starts
            batch = q_starts.numel() - 1
            if batch < 0:
                raise ValueError("starts must hold one more than there are sequences")
            qs, index = _where(q_starts, "q_starts", batch + 1, dev, None)
            ks, index = _where(k_starts, "k_starts", batch + 1, dev, index)
    ql, index = _where(q_lengths, "q_lengths", batch, dev, index)
    kl, index = _where(k_lengths, "k_lengths", batch, dev, index)
    args = _ATTN.pack(batch, n_q, n_k, sq[-2], sk[-2], dim, bool(causal), _type_code(q), I32 if index is None else index, qs, ks, ql, kl,
                      dim ** -0.5 if scale is None else scale)
    return sq, sk, args, hq, hk, hv


def _fresh(like, shape):
    t = like.new_empty(shape)
    heads, dim = shape[-2:]
    return t, _HEADS.pack(t.data_ptr(), shape[-3] * heads * dim, heads * dim, dim)


def attention(q, k, v, q_starts=None, k_starts=None, q_lengths=None, k_lengths=None, causal=True, scale=None, out=None,
              workspace=None, stream=None):
    """softmax(scale * q k^T) v over the keys that a query sees, and the logarithm of the sum of
    the scores' exponentials: (out, lse), out like q and lse float32 [batch, seq, heads]
    or [tokens, heads].

    ``q``             [batch, seq, heads, dim], or [tokens, heads, dim]: one sequence, or
                    several packed ones, sequence s the tokens from ``q_starts[s]`` to
                    ``q_starts[s + 1]`` (int32 or int64, on the device, never decreasing).
    ``k``, ``v``      the same with tokens of their own (a cache) and fewer heads if need be:
                    heads are shared by q_heads / k_heads queries' heads. ``k_starts``
                    are ``q_starts`` unless they are given.
    ``q_lengths``,    tokens in use at the start of each sequence (device; default: all). The
    ``k_lengths``     others are not read: zeros come out.
    ``causal``        the last query in use sees all keys in use, each one before it one less.
                    A query that sees no key gives zeros, and minus infinity for lse.
    ``scale``         dim ** -0.5 by default; positive.

    bfloat16 inputs' probabilities are rounded to bfloat16 for their product with v; float32 inputs keep
    them in float32. The gradients of q, k and v are ``attention_grad``'s."""
    torch = _torch()
    _keeps("attention", scale, q, k, v)
    sq, sk, args, hq, hk, hv = _attn_args(q, k, v, q_starts, k_starts, q_lengths, k_lengths, causal, scale)
    dev = q.device
    if _away(dev, stream):
        return _on(dev, stream, attention, q, k, v, q_starts, k_starts, q_lengths, k_lengths, causal, scale, out, workspace)
    if out is None and (q.requires_grad or k.requires_grad or v.requires_grad) and torch.is_grad_enabled():
        return _functions().Attention.apply(q, k, v, q_starts, k_starts, q_lengths, k_lengths, causal, scale, workspace)
    L = lib()
    held, ws, ws_bytes = _workspace(L.himuon_attention_workspace_size(args), workspace, q)
    if out is None:
        out, ho = _fresh(q, sq)
    else:
        ho = _heads_like(out, "out", sq, q)
    lse = out.new_empty(sq[:-1], dtype=torch.float32)
    _done(L.himuon_attention(args, hq, hk, hv, ho, lse.data_ptr(), ws, ws_bytes, _stream_of(dev.index)), "himuon_attention")
    return out, lse


def attention_grad(g, q, k, v, out, lse, q_starts=None, k_starts=None, q_lengths=None, k_lengths=None, causal=True, scale=None,
                   grads=None, workspace=None, stream=None):
    """The backward pass of ``attention``: from the gradient ``g`` of its result, and its
    inputs and results, (dq, dk, dv). ``grads``: the three tensors to write, which must not overlap."""
    torch = _torch()
    _keeps("attention_grad", scale, g, q, k, v, out, lse)
    sq, sk, args, hq, hk, hv = _attn_args(q, k, v, q_starts, k_starts, q_lengths, k_lengths, causal, scale)
    dev = q.device
    hg, ho = _heads_like(g, "g", sq, q), _heads_like(out, "out", sq, q)
    if lse.shape != sq[:-1] or lse.dtype != torch.float32 or lse.device != dev or not lse.is_contiguous():
        raise ValueError("lse must be attention's: contiguous float32, one value per query and head")
    if _away(dev, stream):
        return _on(dev, stream, attention_grad, g, q, k, v, out, lse, q_starts, k_starts, q_lengths, k_lengths, causal, scale, grads,
                   workspace)
    L = lib()
    held, ws, ws_bytes = _workspace(L.himuon_attention_grad_workspace_size(args), workspace, q)
    if grads is None:
        (dq, gq), (dk, gk), (dv, gv) = _fresh(q, sq), _fresh(k, sk), _fresh(v, sk)
    else:
        dq, dk, dv = grads
        gq, gk, gv = _heads_like(dq, "grads", sq, q), _heads_like(dk, "grads", sk, k), _heads_like(dv, "grads", sk, k)
    _done(L.himuon_attention_grad(args, hg, hq, hk, hv, ho, lse.data_ptr(), gq, gk, gv, ws, ws_bytes, _stream_of(dev.index)),
          "himuon_attention_grad")
    return dq, dk, dv


# ------------------------------------------------------------------ log probabilities

def _logits(logits, tokens):
    """(rows, vocab, leading dimension), checked."""
    rows, vocab, ld = _rows(logits, "logits")
    if tuple(tokens.shape) != tuple(logits.shape[:-1]) or not tokens.is_contiguous():
        raise ValueError("tokens must be a contiguous tensor, one per row of logits")
    _same_device(logits.device, tokens)
    return rows, vocab, ld


def token_logprob(logits, tokens, top=0, scale=1.0, stream=None):
    """Of softmax(scale * logits) over the last dimension: the logarithm of each given
    token's probability, the entropy and the logarithm of the sum of exponentials:
    (logprob, entropy, lse), float32 of ``tokens``' shape; with ``top`` (up to 64) also the
    most likely tokens' log probabilities and indices (int64), [..., top], the
    largest first, equal ones by index.

    ``logits``  [..., vocab], contiguous or 2-D with strided rows.
    ``tokens``  contiguous int32 or int64. One outside the vocabulary (such as -1 for padding) marks
              a row that is not in use: its results are zeros (indices -1).

    The gradient of ``logits`` from those of logprob and entropy is ``token_logprob_grad``'s."""
    torch = _torch()
    _keeps("token_logprob", scale, logits)
    vocab = _logits(logits, tokens)[1]
    dev = logits.device
    _type_code(logits), _index_code(tokens)
    if not 0 <= top <= min(vocab, MAX_TOP):
        raise ValueError(f"top must be between 0 and the smaller of {MAX_TOP} and the vocabulary")
    if _away(dev, stream):
        return _on(dev, stream, token_logprob, logits, tokens, top, scale)
    if logits.requires_grad and torch.is_grad_enabled():
        return _functions().TokenLogprob.apply(logits, tokens, top, scale)
    return _token_logprob(logits, tokens, top, scale, torch.empty((3, *tokens.shape), dtype=torch.float32, device=dev).unbind(0))


def _token_logprob(logits, tokens, top, scale, results):
    """``token_logprob`` into (logprob, entropy, lse); the arguments have been checked."""
    rows, vocab, ld = _rows(logits, "logits")
    logprob, entropy, lse = results
    best = best_index = None
    if top:
        best = lse.new_empty((*tokens.shape, top))
        best_index = lse.new_empty((*tokens.shape, top), dtype=_torch().int64)
    _done(lib().himuon_token_logprob(rows, vocab, logits.data_ptr(), ld, _type_code(logits), tokens.data_ptr(), _index_code(tokens),
                                     scale, top, logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr(),
                                     best.data_ptr() if top else None, best_index.data_ptr() if top else None,
                                     _stream_of(logits.device.index)), "himuon_token_logprob")
    return (logprob, entropy, lse, best, best_index) if top else (logprob, entropy, lse)


def _per_row(t, what, tokens):
    if t is None:
        return None
    if t.shape != tokens.shape or t.dtype != _torch().float32 or t.device != tokens.device or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous float32 tensor of the tokens' shape")
    return t.data_ptr()


def token_logprob_grad(g_logprob, g_entropy, logits, tokens, lse, entropy, scale=1.0, out=None, stream=None):
    """The backward pass of ``token_logprob``: from the gradients of logprob and entropy
    (either may be None), its inputs and its results lse and entropy, the gradient of the
    logits. ``out``: the tensor for it (the logits themselves are allowed)."""
    _keeps("token_logprob_grad", scale, g_logprob, g_entropy, logits, lse, entropy)
    rows, vocab, ld = _logits(logits, tokens)
    dev, code, index = logits.device, _type_code(logits), _index_code(tokens)
    if lse is None or (g_entropy is not None and entropy is None):
        raise ValueError("lse, and entropy where it has a gradient, must be given")
    rest = [_per_row(t, w, tokens) for t, w in ((g_logprob, "g_logprob"), (g_entropy, "g_entropy"), (lse, "lse"), (entropy, "entropy"))]
    if _away(dev, stream):
        return _on(dev, stream, token_logprob_grad, g_logprob, g_entropy, logits, tokens, lse, entropy, scale, out)
    if out is None:
        out, ld_out = logits.new_empty(logits.shape), vocab
    else:
        ld_out = _rows_like(out, "out", logits)
    _done(lib().himuon_token_logprob_grad(rows, vocab, rest[0], rest[1], logits.data_ptr(), ld, code, tokens.data_ptr(), index, rest[2],
                                          rest[3], scale, out.data_ptr(), ld_out, _stream_of(dev.index)), "himuon_token_logprob_grad")
    return out
