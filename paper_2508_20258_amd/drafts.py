"""A step with drafted tokens: a cache of keys and values in bfloat16, appending to it with the rotation on the way, attention of the drafted tokens over it, the
verification of the drafts, and the accepted path kept in the cache.  Same names as the C entry points (include/swz_drafts.h); argument marshalling only, as in
attention_layer.py, whose layouts of heads, `cu`, block tables and meaning of `stream` are these too.

A step's block of tokens of a sequence is its last token that stands (the root) and drafts: a chain, or a tree of up to 64 tokens in which parents stand before children.  A server's step:

    cache16_append(cache, k, v, cu, lengths, table, q=q, cos=cos, sin=sin, positions=lengths_of_tokens + depths)
    out = cache16_attention(q, cache, cu, lengths + counts, table, tree=masks)
    accepted, path, token = verify_drafts(softmax(logits), tokens, cu, uniforms, parents=parents)
    cache16_keep(cache, cu, lengths, path, accepted, table)
    lengths += accepted + 1
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

from .attention_layer import _Heads, _done, _heads, _is_heads, _is_ints, _out, _pointer, _workspace
from .binding import _NoFast, _check, _fast, _launch_stream, _run_on, lib, torch

EXPORTS = ("swz_cache16_append", "swz_cache16_attention_workspace", "swz_cache16_attention", "swz_verify_drafts_workspace", "swz_verify_drafts", "swz_cache16_keep")


class _Cache16(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_tokens", ctypes.c_int32), ("k_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class _AppendArgs(ctypes.Structure):
    _fields_ = [("q", _Heads), ("k", _Heads), ("v", _Heads), ("q_out", _Heads), ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("cu", ctypes.c_void_p), ("before", ctypes.c_void_p), ("block_table", ctypes.c_void_p), ("tokens", ctypes.c_int64), ("table_rows", ctypes.c_int64),
                ("sequences", ctypes.c_int32), ("table_width", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class _DraftAttentionArgs(ctypes.Structure):
    _fields_ = [("q", _Heads), ("out", _Heads), ("cu", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("block_table", ctypes.c_void_p), ("tree", ctypes.c_void_p),
                ("tokens", ctypes.c_int64), ("sequences", ctypes.c_int32), ("table_width", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("max_length", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class _VerifyArgs(ctypes.Structure):
    _fields_ = [("target", ctypes.c_void_p), ("draft", ctypes.c_void_p), ("target_pitch", ctypes.c_int64), ("draft_pitch", ctypes.c_int64), ("vocab", ctypes.c_int64),
                ("total", ctypes.c_int64), ("tokens", ctypes.c_void_p), ("parents", ctypes.c_void_p), ("cu", ctypes.c_void_p), ("uniforms", ctypes.c_void_p),
                ("accepted", ctypes.c_void_p), ("path", ctypes.c_void_p), ("token", ctypes.c_void_p), ("sequences", ctypes.c_int32), ("elem_bytes", ctypes.c_int32)]


def _declare() -> None:
    i32, i64, vp, p = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.POINTER
    lib.swz_cache16_append.argtypes = [p(_Cache16), p(_AppendArgs), vp]
    lib.swz_cache16_attention_workspace.argtypes = [p(_Cache16), p(_DraftAttentionArgs)]
    lib.swz_cache16_attention.argtypes = [p(_Cache16), p(_DraftAttentionArgs), vp, i64, vp]
    lib.swz_verify_drafts_workspace.argtypes = [p(_VerifyArgs)]
    lib.swz_verify_drafts.argtypes = [p(_VerifyArgs), vp, i64, vp]
    lib.swz_cache16_keep.argtypes = [p(_Cache16), vp, vp, vp, vp, i64, vp, i32, i32, vp]
    for name in EXPORTS:
        getattr(lib, name).restype = i64 if name.endswith("_workspace") else ctypes.c_int


_declare()
if _fast is not _NoFast:
    _fast.bind_drafts(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in EXPORTS))


class Cache16(NamedTuple):
    """Keys and values in pages, bfloat16, (pages, k_heads, page_tokens, head_dim) each; `kv_cache16` makes an empty one."""
    k: "torch.Tensor"
    v: "torch.Tensor"


def kv_cache16(pages: int, k_heads: int, head_dim: int, page_tokens: int = 64, device="cuda") -> Cache16:
    """An empty cache.  What is in places that nothing was appended to is not read."""
    assert page_tokens >= 16 and page_tokens & (page_tokens - 1) == 0 and head_dim in (64, 128)
    return Cache16(*(torch.zeros((pages, k_heads, page_tokens, head_dim), dtype=torch.bfloat16, device=device) for _ in range(2)))


def _cache(c: Cache16) -> _Cache16:
    for t in c:
        assert t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous() and t.dim() == 4 and t.shape == c.k.shape
    pages, heads, page, dim = c.k.shape
    return _Cache16(c.k.data_ptr(), c.v.data_ptr(), pages, page, heads, dim)


def _check_blocks(cu, counts, block_table) -> int:
    n = counts.shape[0]
    assert _is_ints(counts, n) and _is_ints(cu, n + 1) and block_table.dim() == 2 and _is_ints(block_table, n, block_table.shape[1])
    return n


def cache16_append(cache: Cache16, k, v, cu, before, block_table, q=None, cos=None, sin=None, positions=None, q_out=None, interleaved: bool = False, stream=None):
    """Token i of sequence b becomes position before[b] + i of it in the cache, the keys turned on the way; returns q turned alike, or None without q.

    k, v (tokens, k_heads, head_dim), q (tokens, q_heads, head_dim); before (sequences,) int32, the tokens already there; block_table (sequences, width) int32, the page of positions
    page_tokens * j .. at [b, j].  cos, sin (rows, rotary_dim / 2) float32 tables; without them nothing is turned, and q is not taken.  positions (tokens,) int32: a row of the tables for each token (in a tree: before[b] and its depth);
    by default its place in the sequence.  A row outside the tables gives NaN.  Pairs are (i, i + rotary_dim / 2), or neighbours with `interleaved`; dimensions from rotary_dim on are not
    turned.  q_out may be q itself.  Positions beyond the table and entries that name no page (-1) are not written.  A page belongs to one sequence of a call."""
    if stream is not None:
        return _run_on(stream, cache16_append, cache, k, v, cu, before, block_table, q, cos, sin, positions, q_out, interleaved)
    if q_out is None:
        done = _fast.cache16_append(cache, k, v, cu, before, block_table, q, cos, sin, positions, interleaved)
        if done is not None:
            return _check(done, "swz_cache16_append") if done.__class__ is int else done
    c = _cache(cache)
    assert _is_heads(k, None, c.k_heads, c.head_dim) and _is_heads(v, *k.shape)
    n, tokens = _check_blocks(cu, before, block_table), k.shape[0]
    a = _AppendArgs(k=_heads(k), v=_heads(v), cu=cu.data_ptr(), before=before.data_ptr(), block_table=block_table.data_ptr(), tokens=tokens, sequences=n,
                    table_width=block_table.shape[1], interleaved=int(bool(interleaved)))
    used = [k, v, cu, before, block_table, *cache]
    assert (cos is None) == (sin is None) and (cos is not None or (q is None and positions is None)) and (q is not None or q_out is None)
    if cos is not None:
        for t in (cos, sin):
            assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.dim() == 2 and t.shape == cos.shape and t.numel() > 0
        a.cos, a.sin, a.rotary_dim, a.table_rows = cos.data_ptr(), sin.data_ptr(), 2 * cos.shape[1], cos.shape[0]
        used += [cos, sin]
    if positions is not None:
        assert _is_ints(positions, tokens)
        a.positions = positions.data_ptr()
        used.append(positions)
    if q is not None:
        assert _is_heads(q, tokens, None, c.head_dim)
        q_out = _out(q_out, q)
        a.q, a.q_out, a.q_heads = _heads(q), _heads(q_out), q.shape[1]
        used += [q, q_out]
    h = _launch_stream(None, *used)
    if tokens > 0:
        _check(lib.swz_cache16_append(ctypes.byref(c), ctypes.byref(a), h), "swz_cache16_append")
    return q_out


def cache16_attention(q, cache: Cache16, cu, lengths, block_table, tree=None, max_length: int = 0, out=None, scale: float | None = None, stream=None):
    """Attention of every sequence's tokens (q: (tokens, q_heads, head_dim), packed) over the first lengths[b] positions of the cache, of which the last are the tokens' own, appended before.

    A token looks at all positions before its block, and at the block's tokens up to itself, or, with `tree` ((tokens,) int64), at token j of its block where bit j is set (draft_tree gives such
    masks); at those from the 65th on none looks then.  A token that looks at nothing gets 0.  A long block (the next piece of a prompt) is right, and costs its products with the whole sequence: `attention` takes a
    third of the time for a prompt by itself.  max_length: the longest length if the program knows it; it decides how sequences are split over the device.
    scale: head_dim ** -0.5 by default."""
    if stream is not None:
        return _run_on(stream, cache16_attention, q, cache, cu, lengths, block_table, tree, max_length, out, scale)
    if out is None:
        done = _fast.cache16_attention(q, cache, cu, lengths, block_table, tree, max_length, scale)
        if done is not None:
            return _done(done, "swz_cache16_attention")
    c = _cache(cache)
    assert _is_heads(q, None, None, c.head_dim)
    n, (tokens, q_heads, dim) = _check_blocks(cu, lengths, block_table), q.shape
    assert tree is None or (tree.is_cuda and tree.dtype == torch.int64 and tree.is_contiguous() and tuple(tree.shape) == (tokens,))
    out = _out(out, q)
    h = _launch_stream(None, q, out, cu, lengths, block_table, *cache, *(() if tree is None else (tree,)))
    if tokens == 0:
        return out
    a = _DraftAttentionArgs(_heads(q), _heads(out), cu.data_ptr(), lengths.data_ptr(), block_table.data_ptr(), _pointer(tree), tokens, n, block_table.shape[1], q_heads, int(max_length),
                            dim ** -0.5 if scale is None else float(scale))
    work = _workspace(lib.swz_cache16_attention_workspace(ctypes.byref(c), ctypes.byref(a)), "swz_cache16_attention", q)
    _check(lib.swz_cache16_attention(ctypes.byref(c), ctypes.byref(a), _pointer(work), 0 if work is None else work.numel(), h), "swz_cache16_attention")
    return out


def verify_drafts(target_probs, tokens, cu, uniforms, draft_probs=None, parents=None, stream=None):
    """(accepted, path, token): which drafts stand and the token after them, so that what is emitted has the target's distribution.

    target_probs (total, vocab), bfloat16 or float32 with dense rows: for each token of the blocks the target's probabilities of what follows it.  tokens (total,) int32 and uniforms (total,) float32 in
    [0, 1): of each node; the root's number is the new token's.  parents (total,) int32: the place in its block of each node's parent, smaller than its own; by default the one before.
    draft_probs, laid out like target_probs: what each node's children were drawn from; without it they may have been chosen by any rule, and a child passes with the target's probability of it.
    accepted (sequences,) int32: how many drafts stand; path (total,) int32: in the place of a block's tokens the places of the root and those drafts, then -1; token (sequences,) int32, -1 where the
    probabilities have no sum.  The exact rule is in include/swz_drafts.h."""
    if stream is not None:
        return _run_on(stream, verify_drafts, target_probs, tokens, cu, uniforms, draft_probs, parents)
    done = _fast.verify_drafts(target_probs, tokens, cu, uniforms, draft_probs, parents)
    if done is not None:
        return _done(done, "swz_verify_drafts")
    used = [target_probs, tokens, cu, uniforms]
    total, vocab = target_probs.shape
    for t in (target_probs, draft_probs):
        if t is not None:
            assert t.is_cuda and t.dtype in (torch.bfloat16, torch.float32) and t.dtype == target_probs.dtype and tuple(t.shape) == (total, vocab)
            assert vocab > 0 and (vocab == 1 or t.stride(1) == 1) and (total < 2 or t.stride(0) >= vocab), "rows are dense and apart"
    assert _is_ints(tokens, total) and cu.dim() == 1 and cu.shape[0] >= 2 and _is_ints(cu, cu.shape[0])
    assert uniforms.is_cuda and uniforms.dtype == torch.float32 and uniforms.is_contiguous() and tuple(uniforms.shape) == (total,)
    if draft_probs is not None:
        used.append(draft_probs)
    if parents is not None:
        assert _is_ints(parents, total)
        used.append(parents)
    n = cu.shape[0] - 1
    h = _launch_stream(None, *used)
    accepted, path, token = (torch.empty(m, dtype=torch.int32, device=cu.device) for m in (n, total, n))
    a = _VerifyArgs(target_pitch=vocab, draft_pitch=vocab, vocab=vocab, total=total, cu=cu.data_ptr(), accepted=accepted.data_ptr(), token=token.data_ptr(), sequences=n,
                    elem_bytes=target_probs.element_size())
    # without tokens nothing of them is read; their tensors have no memory then
    a.target, a.tokens, a.uniforms, a.path = (t.data_ptr() or cu.data_ptr() for t in (target_probs, tokens, uniforms, path))
    if total > 1:
        a.target_pitch = target_probs.stride(0)
    if draft_probs is not None:
        a.draft = draft_probs.data_ptr() or cu.data_ptr()
        if total > 1:
            a.draft_pitch = draft_probs.stride(0)
    if parents is not None:
        a.parents = parents.data_ptr() or cu.data_ptr()
    work = _workspace(lib.swz_verify_drafts_workspace(ctypes.byref(a)), "swz_verify_drafts", cu)
    _check(lib.swz_verify_drafts(ctypes.byref(a), work.data_ptr(), work.numel(), h), "swz_verify_drafts")
    return accepted, path, token


def cache16_keep(cache: Cache16, cu, before, path, accepted, block_table, stream=None) -> None:
    """Keeps the accepted path of every sequence's block, whose tokens were appended after its first before[b] positions: position before[b] + path[cu[b] + i] moves to before[b] + i, i up to
    accepted[b].  path and accepted as verify_drafts returns them (a path rises); the sequences then have before + accepted + 1 positions."""
    if stream is None:
        status = _fast.cache16_keep(cache, cu, before, path, accepted, block_table)
        if status is not None:
            return _check(status, "swz_cache16_keep")
    c = _cache(cache)
    n, total = _check_blocks(cu, before, block_table), path.shape[0]
    assert _is_ints(path, total) and _is_ints(accepted, n)
    h = _launch_stream(stream, cu, before, path, accepted, block_table, *cache)
    if total > 0:
        _check(lib.swz_cache16_keep(ctypes.byref(c), cu.data_ptr(), before.data_ptr(), path.data_ptr(), accepted.data_ptr(), total, block_table.data_ptr(), block_table.shape[1], n, h),
               "swz_cache16_keep")


def draft_tree(parents) -> tuple[list[int], list[int]]:
    """(masks, depths) of a tree of up to 64 tokens, given the place of each one's parent (the root's is not read): for each token the bits of those on its path, itself among them, as the signed 64-bit
    numbers that `tree` of cache16_attention takes, and how far it is from the root.  Plain Python numbers."""
    masks, depths = [], []
    assert len(parents) <= 64
    for i, p in enumerate(parents):
        assert i == 0 or 0 <= p < i, "a parent stands before its children"
        masks.append(1 << i | (masks[p] if i else 0))
        depths.append(depths[p] + 1 if i else 0)
    return [m - (1 << 64) if m >> 63 else m for m in masks], depths
