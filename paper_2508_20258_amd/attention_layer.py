"""Attention layers: norm and rotation of queries and keys, attention over packed prompts with its gradient, and a cache of keys and
values in 4 bits with the attention of single tokens over it.  Same names as the C entry points (include/swz_attention.h); argument
marshalling only, as in binding.py.

Tensors of heads are bfloat16, (tokens, heads, head_dim) with dense head_dim and any distances that are multiples of 8 elements, so that queries, keys and
values may be views of the rows that one projection wrote.  Sequences are packed: `cu` (int32, sequences + 1) holds the first token of each, and the end.

`stream`: what works, with its outputs and workspaces, instead of the current stream.  As for the library's other functions, the caller orders it with the streams that make
the inputs and use the outputs.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

from .binding import _NoFast, _check, _fast, _launch_stream, _run_on, lib, torch

EXPORTS = ("swz_qk_norm_rope", "swz_qk_norm_rope_backward_workspace", "swz_qk_norm_rope_backward", "swz_attention_workspace", "swz_attention", "swz_attention_backward_workspace",
           "swz_attention_backward", "swz_cache4_append", "swz_cache4_read", "swz_cache4_attention_workspace", "swz_cache4_attention")
CACHE_GROUP = 64            # values of a head that share a step and a low


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class _NormArgs(ctypes.Structure):
    _fields_ = [("q", _Heads), ("k", _Heads), ("q_out", _Heads), ("k_out", _Heads), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("tokens", ctypes.c_int64),
                ("q_heads", ctypes.c_int32), ("k_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("table_rows", ctypes.c_int64), ("eps", ctypes.c_float)]


class _AttentionArgs(ctypes.Structure):
    _fields_ = [("q", _Heads), ("k", _Heads), ("v", _Heads), ("out", _Heads), ("lse", ctypes.c_void_p), ("cu_q", ctypes.c_void_p), ("cu_k", ctypes.c_void_p),
                ("total_q", ctypes.c_int64), ("total_k", ctypes.c_int64), ("sequences", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("k_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("causal", ctypes.c_int32), ("scale", ctypes.c_float)]


class _Cache4(ctypes.Structure):
    _fields_ = [("k_words", ctypes.c_void_p), ("v_words", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("pages", ctypes.c_int64), ("page_tokens", ctypes.c_int32), ("k_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


def _declare() -> None:
    i32, i64, vp, f, p = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.POINTER
    h, n, a, c = p(_Heads), p(_NormArgs), p(_AttentionArgs), p(_Cache4)
    lib.swz_qk_norm_rope.argtypes = [n, vp]
    lib.swz_qk_norm_rope_backward_workspace.argtypes = [n]
    lib.swz_qk_norm_rope_backward.argtypes = [n, h, h, vp, vp, vp, i64, vp]
    lib.swz_attention.argtypes = [a, vp, i64, vp]
    lib.swz_attention_workspace.argtypes = lib.swz_attention_backward_workspace.argtypes = [a]
    lib.swz_attention_backward.argtypes = [a, h, h, h, h, vp, i64, vp]
    lib.swz_cache4_append.argtypes = lib.swz_cache4_read.argtypes = [c, h, h, i64, vp, vp, vp, i32, i32, vp]
    lib.swz_cache4_attention_workspace.argtypes = [c, i32, i32, i32, i32]
    lib.swz_cache4_attention.argtypes = [c, h, h, vp, vp, i32, i32, i32, i32, f, vp, i64, vp]
    for name in EXPORTS:
        getattr(lib, name).restype = i64 if name.endswith("_workspace") else ctypes.c_int


_declare()
if _fast is not _NoFast:
    _fast.bind_attention(*(ctypes.cast(getattr(lib, "swz_" + name), ctypes.c_void_p).value for name in (
        "qk_norm_rope", "qk_norm_rope_backward_workspace", "qk_norm_rope_backward", "attention_workspace", "attention", "attention_backward_workspace",
        "attention_backward", "cache4_append", "cache4_read", "cache4_attention_workspace", "cache4_attention")))


def _done(result, where: str):
    """What the ordinary call returned: its result, or the status it failed with."""
    if result.__class__ is int:
        _check(result, where)
    return result


def _heads(t) -> _Heads:
    token, head, _ = t.stride()
    return _Heads(t.data_ptr(), token if t.shape[0] > 1 else 0, head if t.shape[1] > 1 else 0)


def _is_heads(t, tokens=None, heads=None, dim=None) -> bool:
    return (t.is_cuda and t.dtype == torch.bfloat16 and t.dim() == 3 and t.stride(2) == 1 and (tokens is None or t.shape[0] == tokens)
            and (heads is None or t.shape[1] == heads) and (dim is None or t.shape[2] == dim))


def _is_ints(t, *shape) -> bool:
    return t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and tuple(t.shape) == shape


def _out(t, like):
    """An output: `t`, or a new dense tensor; its tokens and heads must not share memory."""
    if t is None:
        return torch.empty(like.shape, dtype=like.dtype, device=like.device)
    assert _is_heads(t, *like.shape)
    (n, h, d), (token, head, _) = t.shape, t.stride()
    assert (n < 2 or h < 2 or token >= h * head >= h * d or head >= n * token >= n * d) and (n < 2 or token >= d) and (h < 2 or head >= d), "tokens or heads of an output overlap"
    return t


def _workspace(size: int, where: str, like):
    if size < 0:
        _check(size, where)
    return torch.empty(size, dtype=torch.uint8, device=like.device) if size else None


def _pointer(t):
    return None if t is None else t.data_ptr()


def _norm_args(q, k, q_out, k_out, q_weight, k_weight, cos, sin, positions, eps, interleaved) -> _NormArgs:
    assert _is_heads(q) and _is_heads(k, q.shape[0], None, q.shape[2])
    tokens, q_heads, dim = q.shape
    for w in (q_weight, k_weight):
        assert w.is_cuda and w.dtype == torch.bfloat16 and w.is_contiguous() and tuple(w.shape) == (dim,)
    for t in (cos, sin):
        assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.dim() == 2 and t.shape == cos.shape
    assert _is_ints(positions, tokens)
    return _NormArgs(_heads(q), _heads(k), _heads(q_out), _heads(k_out), q_weight.data_ptr(), k_weight.data_ptr(), cos.data_ptr(), sin.data_ptr(),
                     positions.data_ptr(), tokens, q_heads, k.shape[1], dim, 2 * cos.shape[1], int(bool(interleaved)), cos.shape[0], float(eps))


def qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions, q_out=None, k_out=None, eps: float = 1e-6, interleaved: bool = False, stream=None):
    """(q_out, k_out): every head of q and k divided by its root mean square (eps under the root), times the weight, and turned by the angles of the token's position.

    q (tokens, q_heads, head_dim), k (tokens, k_heads, head_dim); weights (head_dim,) bfloat16; cos, sin (positions, rotary_dim / 2) float32 tables; positions
    (tokens,) int32.  Pairs are (i, i + rotary_dim / 2), or neighbours with `interleaved`; dimensions from rotary_dim on are not turned.  The outputs may be q and
    k themselves.  A position outside the tables gives NaN."""
    if stream is not None:
        return _run_on(stream, qk_norm_rope, q, k, q_weight, k_weight, cos, sin, positions, q_out, k_out, eps, interleaved)
    if q_out is None and k_out is None:
        done = _fast.qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
        if done is not None:
            return _done(done, "swz_qk_norm_rope")
    q_out, k_out = _out(q_out, q), _out(k_out, k)
    a = _norm_args(q, k, q_out, k_out, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    h = _launch_stream(None, q, k, q_out, k_out, q_weight, k_weight, cos, sin, positions)
    if q.shape[0] > 0:
        _check(lib.swz_qk_norm_rope(ctypes.byref(a), h), "swz_qk_norm_rope")
    return q_out, k_out


def qk_norm_rope_backward(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, positions, dq=None, dk=None, eps: float = 1e-6, interleaved: bool = False, stream=None):
    """(dq, dk, dq_weight, dk_weight) from the gradients of qk_norm_rope's outputs and its inputs; the weights' gradients are float32 sums over all tokens and
    heads.  dq, dk may be dq_out, dk_out themselves."""
    if stream is not None:
        return _run_on(stream, qk_norm_rope_backward, dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, positions, dq, dk, eps, interleaved)
    if dq is None and dk is None:
        done = _fast.qk_norm_rope_backward(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
        if done is not None:
            return _done(done, "swz_qk_norm_rope_backward")
    assert _is_heads(dq_out, *q.shape) and _is_heads(dk_out, *k.shape)
    dq, dk = _out(dq, q), _out(dk, k)
    a = _norm_args(q, k, dq_out, dk_out, q_weight, k_weight, cos, sin, positions, eps, interleaved)
    weights = torch.empty((2, q.shape[2]), dtype=torch.float32, device=q.device)
    h = _launch_stream(None, q, k, dq_out, dk_out, dq, dk, q_weight, k_weight, cos, sin, positions)
    if q.shape[0] == 0:
        return dq, dk, *weights.zero_()
    work = _workspace(lib.swz_qk_norm_rope_backward_workspace(ctypes.byref(a)), "swz_qk_norm_rope_backward", q)
    _check(lib.swz_qk_norm_rope_backward(ctypes.byref(a), ctypes.byref(_heads(dq)), ctypes.byref(_heads(dk)), weights[0].data_ptr(), weights[1].data_ptr(),
                                         work.data_ptr(), work.numel(), h), "swz_qk_norm_rope_backward")
    return dq, dk, weights[0], weights[1]


def _attention_args(q, k, v, out, lse, cu_q, cu_k, causal, scale) -> _AttentionArgs:
    return _AttentionArgs(_heads(q), _heads(k), _heads(v), _heads(out), lse.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(), q.shape[0], k.shape[0],
                          cu_q.shape[0] - 1, q.shape[1], k.shape[1], q.shape[2], int(bool(causal)), q.shape[2] ** -0.5 if scale is None else float(scale))


def _check_prompt(q, k, v, cu_q, cu_k):
    cu_k = cu_q if cu_k is None else cu_k
    assert _is_heads(q) and _is_heads(k, None, None, q.shape[2]) and _is_heads(v, *k.shape)
    assert cu_q.dim() == 1 and cu_q.shape[0] >= 2 and _is_ints(cu_q, cu_q.shape[0]) and _is_ints(cu_k, cu_q.shape[0])
    return cu_k


def attention(q, k, v, cu_q, cu_k=None, out=None, lse=None, causal: bool = True, scale: float | None = None, stream=None):
    """(out, lse): softmax(scale q k^T) v for every sequence and head, and the logarithm of the sum of exponentials, float32 (q_heads, tokens).

    q (tokens, q_heads, head_dim), k and v (key tokens, k_heads, head_dim), q_heads a multiple of k_heads; cu_k where keys belong to other tokens than queries.
    causal: the last query of a sequence looks at all its keys, each before at one fewer.  scale: head_dim ** -0.5 by default."""
    if stream is not None:
        return _run_on(stream, attention, q, k, v, cu_q, cu_k, out, lse, causal, scale)
    if out is None and lse is None:
        done = _fast.attention(q, k, v, cu_q, cu_k, causal, scale)
        if done is not None:
            return _done(done, "swz_attention")
    cu_k = _check_prompt(q, k, v, cu_q, cu_k)
    out = _out(out, q)
    if lse is None:
        lse = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=q.device)
    assert lse.is_cuda and lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == (q.shape[1], q.shape[0])
    h = _launch_stream(None, q, k, v, out, lse, cu_q, cu_k)
    if q.shape[0] == 0:
        return out, lse
    keys = k.shape[0]
    if keys == 0:
        k = v = _of_no_tokens(k, q)
    a = _attention_args(q, k, v, out, lse, cu_q, cu_k, causal, scale)
    a.total_k = keys
    work = _workspace(lib.swz_attention_workspace(ctypes.byref(a)), "swz_attention", q)
    _check(lib.swz_attention(ctypes.byref(a), _pointer(work), 0 if work is None else work.numel(), h), "swz_attention")
    return out, lse


def attention_backward(dout, q, k, v, out, lse, cu_q, cu_k=None, dq=None, dk=None, dv=None, causal: bool = True, scale: float | None = None, stream=None):
    """(dq, dk, dv) from the gradient of attention's out, its arguments and what it returned."""
    if stream is not None:
        return _run_on(stream, attention_backward, dout, q, k, v, out, lse, cu_q, cu_k, dq, dk, dv, causal, scale)
    if dq is None and dk is None and dv is None:
        done = _fast.attention_backward(dout, q, k, v, out, lse, cu_q, cu_k, causal, scale)
        if done is not None:
            return _done(done, "swz_attention_backward")
    cu_k = _check_prompt(q, k, v, cu_q, cu_k)
    assert _is_heads(dout, *q.shape) and _is_heads(out, *q.shape)
    assert lse.is_cuda and lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == (q.shape[1], q.shape[0])
    dq, dk, dv = _out(dq, q), _out(dk, k), _out(dv, v)
    h = _launch_stream(None, dout, q, k, v, out, lse, cu_q, cu_k, dq, dk, dv)
    queries, keys, grads = q.shape[0], k.shape[0], (dq, dk, dv)
    if queries == 0 and keys == 0:
        return grads
    if keys == 0:
        k = v = dk = dv = _of_no_tokens(k, q)
    if queries == 0:
        q = dout = out = dq = _of_no_tokens(q, k)
    a = _attention_args(q, k, v, out, lse, cu_q, cu_k, causal, scale)
    a.total_q, a.total_k, a.lse = queries, keys, a.lse or q.data_ptr()
    work = _workspace(lib.swz_attention_backward_workspace(ctypes.byref(a)), "swz_attention_backward", q)
    _check(lib.swz_attention_backward(ctypes.byref(a), *(ctypes.byref(_heads(t)) for t in (dout, dq, dk, dv)), _pointer(work), 0 if work is None else work.numel(), h),
           "swz_attention_backward")
    return grads


def _of_no_tokens(t, other):
    """In the place of heads of no tokens, which have no memory: a pointer that the library takes, and that nothing is read from or written to."""
    return other[:1, :1].expand(1, t.shape[1], -1)


class Cache4(NamedTuple):
    """Keys and values in pages, 4 bits a value: 64 values of a head share a bfloat16 step and low, value = low + step * n.  Layouts in include/swz_attention.h;
    `kv_cache4` makes an empty one."""
    k_words: "torch.Tensor"       # (pages, k_heads, page_tokens, head_dim / 8) int32
    v_words: "torch.Tensor"       # (pages, k_heads, page_tokens / 8, head_dim) int32
    k_scales: "torch.Tensor"      # (pages, k_heads, page_tokens, head_dim / 64, 2) bfloat16: step, low
    v_scales: "torch.Tensor"


def kv_cache4(pages: int, k_heads: int, head_dim: int, page_tokens: int = 64, device="cuda") -> Cache4:
    """An empty cache.  What is in pages that nothing was appended to is not read."""
    assert page_tokens >= 32 and page_tokens & (page_tokens - 1) == 0 and head_dim in (64, 128)
    words = [torch.zeros(shape, dtype=torch.int32, device=device)
             for shape in ((pages, k_heads, page_tokens, head_dim // 8), (pages, k_heads, page_tokens // 8, head_dim))]
    scales = [torch.zeros((pages, k_heads, page_tokens, head_dim // CACHE_GROUP, 2), dtype=torch.bfloat16, device=device) for _ in range(2)]
    return Cache4(*words, *scales)


def _cache(c: Cache4) -> _Cache4:
    pages, heads, page, words = c.k_words.shape
    dim = 8 * words
    for t, dtype, shape in ((c.k_words, torch.int32, (pages, heads, page, words)), (c.v_words, torch.int32, (pages, heads, page // 8, dim)),
                            (c.k_scales, torch.bfloat16, (pages, heads, page, dim // CACHE_GROUP, 2)),
                            (c.v_scales, torch.bfloat16, (pages, heads, page, dim // CACHE_GROUP, 2))):
        assert t.is_cuda and t.dtype == dtype and t.is_contiguous() and tuple(t.shape) == shape
    return _Cache4(c.k_words.data_ptr(), c.v_words.data_ptr(), c.k_scales.data_ptr(), c.v_scales.data_ptr(), pages, page, heads, dim)


def cache4_append(cache: Cache4, k, v, cu, before, block_table, stream=None) -> None:
    """Token i of sequence b becomes position before[b] + i of it in the cache.

    k, v (tokens, k_heads, head_dim); before (sequences,) int32, the tokens already there; block_table (sequences, width) int32, the page of positions page_tokens * j ..
    at [b, j].  Positions beyond the table and entries that name no page (-1) are not written.  A page belongs to one sequence of a call."""
    if stream is None:
        status = _fast.cache4_append(cache, k, v, cu, before, block_table)
        if status is not None:
            return _check(status, "swz_cache4_append")
    c = _cache(cache)
    assert _is_heads(k, None, c.k_heads, c.head_dim) and _is_heads(v, *k.shape)
    n = before.shape[0]
    assert _is_ints(before, n) and _is_ints(cu, n + 1) and block_table.dim() == 2 and _is_ints(block_table, n, block_table.shape[1])
    h = _launch_stream(stream, k, v, cu, before, block_table, *cache)
    if k.shape[0] > 0:
        _check(lib.swz_cache4_append(ctypes.byref(c), ctypes.byref(_heads(k)), ctypes.byref(_heads(v)), k.shape[0], cu.data_ptr(), before.data_ptr(),
                                     block_table.data_ptr(), block_table.shape[1], n, h), "swz_cache4_append")


def cache4_read(cache: Cache4, cu, first, block_table, tokens: int, k=None, v=None, stream=None):
    """(k, v): positions first[b] .. of every sequence, cu[b + 1] - cu[b] of them, as bfloat16 (tokens, k_heads, head_dim); tokens is cu's last entry."""
    if stream is not None:
        return _run_on(stream, cache4_read, cache, cu, first, block_table, tokens, k, v)
    if k is None and v is None:
        done = _fast.cache4_read(cache, cu, first, block_table, tokens)
        if done is not None:
            return _done(done, "swz_cache4_read")
    c = _cache(cache)
    n = first.shape[0]
    assert _is_ints(first, n) and _is_ints(cu, n + 1) and block_table.dim() == 2 and _is_ints(block_table, n, block_table.shape[1])
    shape = (int(tokens), c.k_heads, c.head_dim)
    like = torch.empty(shape, dtype=torch.bfloat16, device="meta") if k is None or v is None else k
    k = torch.empty(shape, dtype=torch.bfloat16, device=cu.device) if k is None else _out(k, like)
    v = torch.empty(shape, dtype=torch.bfloat16, device=cu.device) if v is None else _out(v, like)
    assert tuple(k.shape) == tuple(v.shape) == shape
    h = _launch_stream(None, k, v, cu, first, block_table, *cache)
    if shape[0] > 0:
        _check(lib.swz_cache4_read(ctypes.byref(c), ctypes.byref(_heads(k)), ctypes.byref(_heads(v)), shape[0], cu.data_ptr(), first.data_ptr(),
                                   block_table.data_ptr(), block_table.shape[1], n, h), "swz_cache4_read")
    return k, v


def cache4_attention(q, cache: Cache4, lengths, block_table, max_length: int = 0, out=None, scale: float | None = None, stream=None):
    """Attention of one token of each sequence (q: (sequences, q_heads, head_dim)) over the first lengths[b] positions of the cache, its own appended before.
    A sequence of length 0 gets 0.  max_length: the longest length if the program knows it; it decides how sequences are split over the device."""
    if stream is not None:
        return _run_on(stream, cache4_attention, q, cache, lengths, block_table, max_length, out, scale)
    if out is None:
        done = _fast.cache4_attention(q, cache, lengths, block_table, max_length, scale)
        if done is not None:
            return _done(done, "swz_cache4_attention")
    c = _cache(cache)
    assert _is_heads(q, None, None, c.head_dim)
    n, q_heads, dim = q.shape
    assert _is_ints(lengths, n) and block_table.dim() == 2 and _is_ints(block_table, n, block_table.shape[1])
    out = _out(out, q)
    h = _launch_stream(None, q, out, lengths, block_table, *cache)
    if n == 0:
        return out
    width, longest = block_table.shape[1], int(max_length)
    work = _workspace(lib.swz_cache4_attention_workspace(ctypes.byref(c), n, q_heads, width, longest), "swz_cache4_attention", q)
    _check(lib.swz_cache4_attention(ctypes.byref(c), ctypes.byref(_heads(q)), ctypes.byref(_heads(out)), lengths.data_ptr(), block_table.data_ptr(), width, n, q_heads,
                                    longest, dim ** -0.5 if scale is None else float(scale), _pointer(work), 0 if work is None else work.numel(), h),
           "swz_cache4_attention")
    return out
