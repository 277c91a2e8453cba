"""Attention with modified scores, and attention of a batch that shares a prefix.

``attention_scored`` computes, with ``x = scale q.k`` and positions ``pos_i = q_pos[b] + i``
of query i and j of key j,

    y = softcap tanh(x / softcap)                                  (``softcap``)
    s = y - slopes[h] |pos_i - j| + bias[bucket(j - pos_i), h]     (``slopes``, ``bias``)
    o_i = sum_j softmax_j(s_ij) v_j                                over the visible keys

where key j is visible to query i if ``j < kv_len[b]``; with ``causal`` if ``j <= pos_i`` or
``j < prefix_len[b]``; and with ``docs`` if both are of the same document.  Everything is
computed tile by tile in the HIP kernels of ``libmea.so`` (nothing of the size of the score
matrix is ever in memory, the bias included), forward and backward, with a gradient for q, k, v
and the bias.  A query that sees no key gets o = 0, lse = -inf and zero gradients.

``q`` is ``[B, H, n_q, d]``, ``k`` and ``v`` are ``[B, H_kv, n_k, d]`` with H a multiple of
H_kv (query head h reads key head ``h // (H // H_kv)``), d 64 or 128, float32, float16 or
bfloat16, any batch, head and row strides that are multiples of 16 bytes.
"""
from __future__ import annotations

import ctypes
import functools
import math

import torch
from torch.autograd.function import once_differentiable

from . import _lib
from .attention import _DTYPE_CODE, _check_tensors, _feature_contiguous, _stream


@functools.lru_cache(maxsize=None)
def bucket_edges(buckets: int, max_distance: int) -> tuple:
    """Smallest distance of each of one side's ``buckets``: a bucket for every distance
    below h = buckets // 2, then bucket b from ``h (max_distance / h)^((b - h) / (buckets - h))``
    on, in whole numbers (no rounding decides a bucket)."""
    h = buckets // 2
    if buckets < 2 or max_distance <= h:
        raise ValueError("a side needs at least 2 buckets and a max_distance above half their number, got %d and %d"
                         % (buckets, max_distance))
    edges = list(range(h))
    for b in range(h, buckets):
        # x >= h (m / h)^(t / n) as x^n >= m^t h^(n - t), from a little below the estimate on.
        n, t = buckets - h, b - h
        x = max(h, int(h * (max_distance / h) ** (t / n)) - 2)
        bound = max_distance ** t * h ** (n - t)
        while x ** n < bound:
            x += 1
        edges.append(x)
    return tuple(edges)


@functools.lru_cache(maxsize=None)
def _side(buckets: int, two_sided: bool, max_distance: int):
    """The edges of a side as a C array."""
    if buckets < 2 or (two_sided and buckets % 2):
        raise ValueError("bias must have at least 2 buckets, an even number if bidirectional, got %d" % buckets)
    edges = bucket_edges(buckets // 2 if two_sided else buckets, max_distance)
    if len(edges) > _lib.MAX_SIDE_BUCKETS or edges[-1] > _lib.MAX_BIAS_SPAN:
        raise ValueError("at most %d buckets a side, the last from at most %d on: got %d, from %d on"
                         % (_lib.MAX_SIDE_BUCKETS, _lib.MAX_BIAS_SPAN, len(edges), edges[-1]))
    return (ctypes.c_int32 * len(edges))(*edges)


@functools.lru_cache(maxsize=None)
def _side_arg(buckets: int, two_sided: bool, max_distance: int):
    """The same for the native calls: address, number and whether there are two sides."""
    edges = _side(buckets, two_sided, max_distance)
    return ctypes.addressof(edges), len(edges), two_sided


def _native_score(causal, softcap, slopes, bias, max_distance, bidirectional, docs, prefix_len, q_pos):
    """The native calls' last arguments, or None where only the general path can say what
    is wrong."""
    if prefix_len is not None and not causal:
        return None
    side = None
    if bias is not None:
        if not isinstance(bias, torch.Tensor) or bias.dim() != 2:
            return None
        side = _side_arg(bias.shape[0], not causal if bidirectional is None else bool(bidirectional), int(max_distance))
    q_doc, k_doc = docs if isinstance(docs, tuple) and len(docs) == 2 else (docs, docs)
    return softcap, slopes, bias, side, q_doc, k_doc, prefix_len, q_pos


def _int32(name, t, shape, device):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32 or t.device != device or tuple(t.shape) != shape \
            or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 %s tensor on q's device" % (name, list(shape)))
    return t


def _shapes(q, k, v):
    if not all(isinstance(t, torch.Tensor) and t.dim() == 4 for t in (q, k, v)):
        raise ValueError("q, k and v must be [B, H, n, d]")
    if q.dtype not in _DTYPE_CODE:
        raise TypeError("unsupported dtype %s" % q.dtype)
    if k.shape != v.shape or q.shape[0] != k.shape[0] or q.shape[3] != k.shape[3] or k.shape[1] < 1 \
            or q.shape[1] % k.shape[1]:
        raise ValueError("shape mismatch: q %s k %s v %s" % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))


def _strides(tensors: dict) -> dict | None:
    """Strides for the ABI where a tensor is not contiguous; those of dimensions of one
    element, which say nothing, are replaced by valid ones."""
    if all(t.is_contiguous() for t in tensors.values()):
        return None
    return {n: tuple(s if size > 1 else t.shape[3] for s, size in zip(t.stride()[:3], t.shape[:3]))
            for n, t in tensors.items()}


def _problem(q, k, causal, scale, kv_len, tensors):
    B, H, n_q, d = q.shape
    _int32("kv_len", kv_len, (B,), q.device)
    return _lib.problem(B, H, n_q, k.shape[2], d, _DTYPE_CODE[q.dtype], causal, 1.0 / math.sqrt(d) if scale is None else scale,
                        False, _strides(tensors), kv_len.data_ptr() if kv_len is not None else None)


def _score(q, k, causal, softcap, slopes, bias, max_distance, bidirectional, docs, prefix_len, q_pos):
    B, H, n_q, _ = q.shape
    s = _lib.MeaScore()
    s.kv_heads = k.shape[1]
    if softcap is not None:
        if not (isinstance(softcap, (int, float)) and softcap > 0 and math.isfinite(softcap)):
            raise ValueError("softcap must be positive and finite, got %r" % (softcap,))
        s.softcap = softcap
    if slopes is not None:
        if not isinstance(slopes, torch.Tensor) or slopes.dtype != torch.float32 or slopes.device != q.device or tuple(slopes.shape) != (H,) or not slopes.is_contiguous():
            raise ValueError("slopes must be a contiguous float32 [H] tensor on q's device")
        s.slopes = slopes.data_ptr()
    if bias is not None:
        if not isinstance(bias, torch.Tensor) or bias.dtype not in (torch.float32, q.dtype) or bias.device != q.device or bias.dim() != 2 or bias.shape[1] != H \
                or not bias.is_contiguous():
            raise ValueError("bias must be a contiguous [buckets, H] tensor on q's device, in float32 or q's dtype")
        two_sided = not causal if bidirectional is None else bool(bidirectional)
        s.edges = _side(bias.shape[0], two_sided, int(max_distance))
        s.n_edges, s.two_sided = bias.shape[0] // (2 if two_sided else 1), two_sided
        s.table, s.table_dtype = bias.data_ptr(), _DTYPE_CODE[bias.dtype]
    if docs is not None:
        if not isinstance(docs, torch.Tensor) and len(docs) != 2:
            raise ValueError("docs must be a tensor, or a pair of those of the queries and of the keys")
        if isinstance(docs, torch.Tensor):
            if n_q != k.shape[2]:
                raise ValueError("docs must be a pair of [B, n_q] and [B, n_k] tensors where n_q and n_k differ")
            docs = (docs, docs)
        s.q_doc = _int32("docs of the queries", docs[0], (B, n_q), q.device).data_ptr()
        s.k_doc = _int32("docs of the keys", docs[1], (B, k.shape[2]), q.device).data_ptr()
    if prefix_len is not None:
        if not causal:
            raise ValueError("prefix_len needs causal=True (without it every key is visible)")
        s.prefix_len = _int32("prefix_len", prefix_len, (B,), q.device).data_ptr()
    if q_pos is not None:
        s.q_pos = _int32("q_pos", q_pos, (B,), q.device).data_ptr()
    return s


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _workspace(size, device):
    return torch.empty(size, dtype=torch.uint8, device=device) if size else None


def attention_scored_fwd(q, k, v, causal: bool = False, scale: float | None = None, need_lse: bool = True, out=None,
                         kv_len=None, residual: bool = False, *, softcap: float | None = None, slopes=None, bias=None,
                         max_distance: int = 128, bidirectional: bool | None = None, docs=None, prefix_len=None, q_pos=None):
    """Returns ``(o, lse)``, or ``(o, lse, o_lo)`` with ``residual`` (see ``attention_fwd``).

    ``softcap``: a positive number.  ``slopes``: float32 ``[H]`` on the GPU, no gradient.  ``bias``:
    ``[buckets, H]`` (float32 or q's dtype), whose bucket of a distance is that of ``bucket_edges``;
    ``bidirectional`` (default: not ``causal``) gives each direction half the buckets, else keys
    ahead count as distance 0; a value of -inf hides its pairs.  ``docs``: int32 ``[B, n]`` document of every token, negative for
    none, or a pair of those of the queries and of the keys.  ``prefix_len``, ``q_pos`` (position of
    the first query; 0 without it, negative values read as 0) and ``kv_len``: int32 ``[B]``.  For a
    step of decoding against a cache, ``q_pos = kv_len - n_q``."""
    mods = _native_score(causal, softcap, slopes, bias, max_distance, bidirectional, docs, prefix_len, q_pos)
    if mods is not None:
        r = _lib.native().scored_fwd(q, k, v, causal, scale, need_lse, out, kv_len, residual, *mods)
        if r is not None:
            return r
    _shapes(q, k, v)
    _check_tensors(("q", "k", "v"), (q, k, v), q.dtype, q.device)
    s = _score(q, k, causal, softcap, slopes, bias, max_distance, bidirectional, docs, prefix_len, q_pos)
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
    _check_tensors(("out",), (o,), q.dtype, q.device)
    if o.shape != q.shape:
        raise ValueError("out must be [B, H, n_q, d]")
    p = _problem(q, k, causal, scale, kv_len, {"q": q, "k": k, "v": v, "o": o})
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if need_lse else None
    o_lo = torch.empty(q.shape, dtype=q.dtype, device=q.device) if residual and q.dtype != torch.float32 else None
    size = _lib.scored_fwd_workspace_size(p, s)
    ws = _workspace(size, q.device)
    with torch.cuda.device(q.device):
        _lib.check("mea_scored_attention_fwd", _lib.scored_fwd(
            p, s, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), _ptr(lse), _ptr(o_lo), _ptr(ws), size,
            _stream(q.device)))
    return (o, lse, o_lo) if residual else (o, lse)


def attention_scored_bwd(q, k, v, o, lse, do, causal: bool = False, scale: float | None = None, need_dq: bool = True,
                         need_dkdv: bool = True, need_dbias: bool = True, kv_len=None, o_lo=None, *,
                         softcap: float | None = None, slopes=None, bias=None, max_distance: int = 128,
                         bidirectional: bool | None = None, docs=None, prefix_len=None, q_pos=None):
    """Returns ``(dq, dk, dv, dbias)`` for the upstream gradient ``do`` of a forward with the
    same arguments; those not needed (and dbias without a bias) are None."""
    mods = _native_score(causal, softcap, slopes, bias, max_distance, bidirectional, docs, prefix_len, q_pos)
    if mods is not None:
        r = _lib.native().scored_bwd(q, k, v, o, lse, do, causal, scale, need_dq, need_dkdv, need_dbias, kv_len, o_lo, *mods)
        if r is not None:
            return r
    _shapes(q, k, v)
    _check_tensors(("q", "k", "v", "o", "do"), (q, k, v, o, do), q.dtype, q.device)
    _check_tensors(("lse",), (lse,), torch.float32, q.device)
    if o.shape != q.shape or do.shape != q.shape or lse.shape != q.shape[:3]:
        raise ValueError("o, do must be [B, H, n_q, d] and lse [B, H, n_q]")
    if o_lo is not None:
        _check_tensors(("o_lo",), (o_lo,), q.dtype, q.device)
        if o_lo.shape != q.shape or not o_lo.is_contiguous():
            raise ValueError("o_lo must be a contiguous [B, H, n_q, d] tensor")
    need_dbias = need_dbias and bias is not None
    if not (need_dq or need_dkdv or need_dbias):
        raise ValueError("nothing to compute")
    s = _score(q, k, causal, softcap, slopes, bias, max_distance, bidirectional, docs, prefix_len, q_pos)
    # The bias's gradient comes out of the dQ kernel.
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if need_dq or need_dbias else None
    dk, dv = (torch.empty(k.shape, dtype=k.dtype, device=k.device) if need_dkdv else None for _ in range(2))
    dbias = torch.empty(bias.shape, dtype=bias.dtype, device=bias.device) if need_dbias else None
    given = {"q": q, "k": k, "v": v, "o": o, "d_o": do, "dq": dq, "dk": dk, "dv": dv}
    p = _problem(q, k, causal, scale, kv_len, {n: t for n, t in given.items() if t is not None})
    size = _lib.scored_bwd_workspace_size(p, s)
    ws = _workspace(size, q.device)
    with torch.cuda.device(q.device):
        _lib.check("mea_scored_attention_bwd", _lib.scored_bwd(
            p, s, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), _ptr(o_lo), do.data_ptr(), lse.data_ptr(),
            _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dbias), _ptr(ws), size, _stream(q.device)))
    return dq if need_dq else None, dk, dv, dbias


class ScoredAttention(torch.autograd.Function):
    """Autograd wrapper of what the native call leaves (copies to readable layouts, errors): saves
    q, k, v, o, the O(n) lse and, for a 16-bit o, its rounding residual."""

    @staticmethod
    def forward(ctx, q, k, v, bias, causal, scale, kv_len, softcap, slopes, max_distance, bidirectional, docs, prefix_len,
                q_pos):
        q, k, v = (_feature_contiguous(t) for t in (q, k, v))
        bias = bias.contiguous() if bias is not None else None
        pair = docs if isinstance(docs, tuple) else (docs, docs)
        o, lse, o_lo = attention_scored_fwd(q, k, v, causal, scale, True, None, kv_len, True, softcap=softcap, slopes=slopes,
                                            bias=bias, max_distance=max_distance, bidirectional=bidirectional, docs=docs,
                                            prefix_len=prefix_len, q_pos=q_pos)
        ctx.save_for_backward(q, k, v, o, lse, o_lo, bias, slopes, *pair, prefix_len, q_pos, kv_len)
        ctx.args = (causal, scale, softcap, max_distance, bidirectional)
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        q, k, v, o, lse, o_lo, bias, slopes, q_doc, k_doc, prefix_len, q_pos, kv_len = ctx.saved_tensors
        causal, scale, softcap, max_distance, bidirectional = ctx.args
        need = ctx.needs_input_grad
        grads = attention_scored_bwd(q, k, v, o, lse, _feature_contiguous(do), causal, scale, need[0], need[1] or need[2],
                                     need[3], kv_len, o_lo, softcap=softcap, slopes=slopes, bias=bias,
                                     max_distance=max_distance, bidirectional=bidirectional,
                                     docs=None if q_doc is None else (q_doc, k_doc), prefix_len=prefix_len, q_pos=q_pos)
        return (*grads, *[None] * 10)


def attention_scored(q, k, v, causal: bool = False, scale: float | None = None, kv_len=None, *, softcap: float | None = None,
                     slopes=None, bias=None, max_distance: int = 128, bidirectional: bool | None = None, docs=None,
                     prefix_len=None, q_pos=None):
    """Attention with modified scores, differentiable in q, k, v and bias, O(n) extra memory;
    the arguments are those of ``attention_scored_fwd``.  Captured into a graph with its gradient,
    it is refused while a graph of the same leaves that was recorded on another stream lives."""
    if slopes is not None and slopes.requires_grad:
        raise ValueError("slopes get no gradient: pass them detached")
    docs = tuple(docs) if isinstance(docs, list) else docs
    mods = _native_score(causal, softcap, slopes, bias, max_distance, bidirectional, docs, prefix_len, q_pos)
    if mods is not None:
        r = _lib.native().scored_apply(q, k, v, causal, scale, kv_len, *mods)
        if r is not None:
            return r
    return ScoredAttention.apply(q, k, v, bias, causal, scale, kv_len, softcap, slopes, max_distance, bidirectional, docs,
                                 prefix_len, q_pos)


def _prefix_strides(name, t):
    """Head and row strides of a ``[H_kv, n_p, d]`` prefix (of one row: any valid row stride)."""
    head, row = (s if size > 1 else t.shape[2] for s, size in zip(t.stride()[:2], t.shape[:2]))
    if row < t.shape[2]:  # (the ABI reads a row stride of 0 as contiguous)
        raise ValueError("the rows of %s overlap: strides %s" % (name, t.stride()))
    return _lib.MeaTensorStrides(0, head, row)


def attention_shared_prefix(q, k_prefix, v_prefix, k, v, causal: bool = False, scale: float | None = None, kv_len=None, *,
                            q_pos=None, out=None, need_lse: bool = False):
    """Attention of a batch whose sequences begin with the same keys: every query sees all of
    ``k_prefix``, ``v_prefix`` (``[H_kv, n_p, d]``, once for the batch) and its own sequence's ``k``,
    ``v`` (``[B, H_kv, n_k, d]``) as ``kv_len`` and ``causal`` with ``q_pos`` say (positions count the
    own keys).  The prefix is read once for all queries of a key head.  Returns o, or ``(o, lse)``
    with ``need_lse``.  For serving: no gradient."""
    if torch.is_grad_enabled() and any(t.requires_grad for t in (q, k_prefix, v_prefix, k, v)):
        raise ValueError("attention_shared_prefix has no gradient: call it under torch.no_grad()")
    r = _lib.native().prefix_fwd(q, k_prefix, v_prefix, k, v, causal, scale, kv_len, q_pos, out, need_lse)
    if r is not None:
        return r if need_lse else r[0]
    _shapes(q, k, v)
    if k_prefix.dim() != 3 or k_prefix.shape != v_prefix.shape or k_prefix.shape[0] != k.shape[1] \
            or k_prefix.shape[2] != q.shape[3]:
        raise ValueError("k_prefix and v_prefix must be [H_kv, n_p, d], got %s and %s"
                         % (tuple(k_prefix.shape), tuple(v_prefix.shape)))
    kp, vp = k_prefix[None], v_prefix[None]
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
    _check_tensors(("q", "k", "v", "k_prefix", "v_prefix", "out"), (q, k, v, kp, vp, o), q.dtype, q.device)
    if o.shape != q.shape:
        raise ValueError("out must be [B, H, n_q, d]")
    p = _problem(q, k, causal, scale, kv_len, {"q": q, "k": k, "v": v, "o": o})
    x = _lib.MeaSharedPrefix()
    x.kv_heads, x.n_p, x.k, x.v = k.shape[1], kp.shape[2], kp.data_ptr(), vp.data_ptr()
    x.k_strides, x.v_strides = _prefix_strides("k_prefix", k_prefix), _prefix_strides("v_prefix", v_prefix)
    if q_pos is not None:
        x.q_pos = _int32("q_pos", q_pos, (q.shape[0],), q.device).data_ptr()
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if need_lse else None
    size = _lib.prefix_fwd_workspace_size(p, x)
    ws = _workspace(size, q.device)
    with torch.cuda.device(q.device):
        _lib.check("mea_prefix_attention_fwd", _lib.prefix_fwd(
            p, x, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), _ptr(lse), _ptr(ws), size, _stream(q.device)))
    return (o, lse) if need_lse else o
