"""The attention oracle against closed forms and differences, and the host side of the attention entry points: exports, refusals.  No GPU."""
import ctypes
import os
import re

import numpy as np
import pytest

import paper_2508_20258_amd as swz
from oracle import attention_ref as ar
from paper_2508_20258_amd import attention_layer as layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_entry_point():
    header = open(os.path.join(ROOT, "include", "swz_attention.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(swz_[a-z0-9_]+)\s*\(", header))
    assert declared == set(layer.EXPORTS)
    raw = ctypes.CDLL(swz.binding.LIB_PATH)
    for name in declared:
        assert hasattr(raw, name), name


def difference(f, x, dz, h=1e-6):
    """Gradient of sum(f(x) * dz) by central differences."""
    g = np.zeros(x.shape)
    for i in np.ndindex(*x.shape):
        y = x.copy()
        y[i] += h
        up = (f(y) * dz).sum()
        y[i] -= 2 * h
        g[i] = (up - (f(y) * dz).sum()) / (2 * h)
    return g


@pytest.mark.parametrize("nq,nk,causal", [(1, 1, True), (5, 5, True), (3, 6, True), (6, 3, True), (4, 7, False)])
def test_attention_gradient_against_differences(nq, nk, causal):
    rng = np.random.default_rng(nq * 10 + nk)
    q, k, v, g = (rng.normal(size=(n, 4)) for n in (nq, nk, nk, nq))
    (dq, dk, dv), _ = ar.attention_backward(q, k, v, 0.5, causal, g)
    for got, want in ((dq, difference(lambda x: ar.attention(x, k, v, 0.5, causal)[0], q, g)), (dk, difference(lambda x: ar.attention(q, x, v, 0.5, causal)[0], k, g)),
                      (dv, difference(lambda x: ar.attention(q, k, x, 0.5, causal)[0], v, g))):
        assert np.allclose(got, want, atol=1e-8)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("r", [2, 4, 8])
def test_norm_gradient_against_differences(interleaved, r):
    rng = np.random.default_rng(r)
    x, dz, w, a = rng.normal(size=(3, 8)), rng.normal(size=(3, 8)), rng.normal(size=8), rng.normal(size=r // 2)
    dx, dw = ar.norm_rope_backward(dz, x, w, np.cos(a), np.sin(a), interleaved, 1e-3)
    assert np.allclose(dx, difference(lambda y: ar.norm_rope(y, w, np.cos(a), np.sin(a), interleaved, 1e-3), x, dz), atol=1e-8)
    assert np.allclose(dw, difference(lambda y: ar.norm_rope(x, y, np.cos(a), np.sin(a), interleaved, 1e-3), w, dz), atol=1e-8)


def test_attention_closed_forms():
    v = np.arange(12.0).reshape(3, 4)
    out, lse, p, _ = ar.attention(np.zeros((3, 4)), np.ones((3, 4)), v, 1.0, True)
    assert np.allclose(out, [v[0], v[:2].mean(0), v.mean(0)]) and np.allclose(lse, np.log([1, 2, 3]))        # equal scores
    out, lse, p, _ = ar.attention(np.ones((3, 4)), np.ones((1, 4)), v[:1], 1.0, True)
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.allclose(out[2], v[0])                 # rows that look at nothing
    out, _, _, _ = ar.attention(np.full((1, 4), 100.0), np.vstack([np.zeros((2, 4)), np.ones((1, 4))]), v, 1.0, False)
    assert np.allclose(out[0], v[2])                                                                          # one score far above


def test_quantise():
    x = np.linspace(-3, 4.5, 64, dtype=np.float32)
    step, low, n = ar.quantise(x)
    assert step == 0.5 and low == -3 and n.min() == 0 and n.max() == 15 and np.abs(low + step * n - x).max() <= 0.25
    assert ar.quantise(np.full(64, 2.5))[0] == 0 and (ar.quantise(np.full(64, 2.5))[2] == 0).all()
    for bad in (np.nan, np.inf, -np.inf):
        y = x.copy()
        y[7] = bad
        assert np.isnan(ar.quantise(y)[0]) and np.isnan(ar.quantise(y)[1])
    assert ar.word([1, 0, 0, 0, 0, 0, 0, 0]) == 1 and ar.word([0, 1, 0, 0, 0, 0, 0, 0]) == 1 << 16 and ar.word([15] * 8) == 0xffffffff
    assert [float(ar.to_bf16(x)) for x in (1.0, 1 + 2 ** -8, 1 + 3 * 2 ** -8)] == [1.0, 1.0, 1 + 2 ** -6]


# ---------------------------------------------------------------- refusals: pointers that are never used

P = 0x1000


def heads(token=256, head=128, data=P):
    return layer._Heads(data, token, head)


def norm_args(**change):
    a = dict(q=heads(), k=heads(), q_out=heads(), k_out=heads(), q_weight=P, k_weight=P, cos=P, sin=P, positions=P, tokens=3, q_heads=2, k_heads=1, head_dim=128,
             rotary_dim=128, interleaved=0, table_rows=10, eps=1e-6)
    a.update(change)
    return layer._NormArgs(*(a[n] for n, _ in layer._NormArgs._fields_))


def prompt_args(**change):
    a = dict(q=heads(), k=heads(), v=heads(), out=heads(), lse=P, cu_q=P, cu_k=P, total_q=3, total_k=3, sequences=1, q_heads=2, k_heads=1, head_dim=128, causal=1, scale=0.1)
    a.update(change)
    return layer._AttentionArgs(*(a[n] for n, _ in layer._AttentionArgs._fields_))


def cache_args(**change):
    a = dict(k_words=P, v_words=P, k_scales=P, v_scales=P, pages=4, page_tokens=64, k_heads=1, head_dim=128)
    a.update(change)
    return layer._Cache4(*(a[n] for n, _ in layer._Cache4._fields_))


INVALID, UNSUPPORTED, OVERFLOW = -1, -2, -3
BAD_HEADS = [(heads(data=None), INVALID), (heads(token=-8), INVALID), (heads(token=4), UNSUPPORTED), (heads(head=132), UNSUPPORTED), (heads(data=P + 2), UNSUPPORTED)]


@pytest.mark.parametrize("change,status", [(dict(q=h), s) for h, s in BAD_HEADS] + [(dict(k_out=h), s) for h, s in BAD_HEADS] + [
    (dict(positions=None), INVALID), (dict(cos=None), INVALID), (dict(k_weight=None), INVALID), (dict(tokens=-1), INVALID), (dict(q_heads=0), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(table_rows=-1), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(rotary_dim=8), UNSUPPORTED),
    (dict(rotary_dim=144), UNSUPPORTED), (dict(rotary_dim=40), UNSUPPORTED), (dict(sin=P + 4), UNSUPPORTED), (dict(tokens=1 << 31), OVERFLOW), (dict(tokens=1 << 30), OVERFLOW)])
def test_norm_refusals(change, status):
    a = norm_args(**change)
    assert layer.lib.swz_qk_norm_rope(ctypes.byref(a), None) == status
    assert layer.lib.swz_qk_norm_rope_backward_workspace(ctypes.byref(a)) == status
    assert layer.lib.swz_qk_norm_rope_backward(ctypes.byref(a), ctypes.byref(heads()), ctypes.byref(heads()), P, P, P, 1 << 40, None) == status


def test_norm_backward_refusals():
    a, h = norm_args(), heads()
    call = lambda dq=h, dk=h, wq=P, wk=P, work=P, size=1 << 40: layer.lib.swz_qk_norm_rope_backward(
        ctypes.byref(a), dq if dq is None else ctypes.byref(dq), dk if dk is None else ctypes.byref(dk), wq, wk, work, size, None)
    need = layer.lib.swz_qk_norm_rope_backward_workspace(ctypes.byref(a))
    assert need > 0
    assert call(dq=None) == call(wk=None) == call(work=None) == call(size=need - 1) == INVALID
    assert call(work=P + 8) == call(dk=heads(token=12)) == UNSUPPORTED
    assert layer.lib.swz_qk_norm_rope(ctypes.byref(norm_args(tokens=0)), None) == 0 and layer.lib.swz_qk_norm_rope(None, None) == INVALID


@pytest.mark.parametrize("change,status", [(dict(q=h), s) for h, s in BAD_HEADS] + [(dict(v=h), s) for h, s in BAD_HEADS] + [
    (dict(lse=None), INVALID), (dict(cu_q=None), INVALID), (dict(sequences=0), INVALID), (dict(q_heads=3, k_heads=2), INVALID), (dict(k_heads=0), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(total_q=-1), INVALID),
    (dict(head_dim=32), UNSUPPORTED), (dict(cu_k=P + 2), UNSUPPORTED), (dict(total_k=1 << 31), OVERFLOW), (dict(total_q=(1 << 31) - 1, q_heads=1024, k_heads=1024), OVERFLOW)])
def test_attention_refusals(change, status):
    a, h = prompt_args(**change), ctypes.byref(heads())
    assert layer.lib.swz_attention(ctypes.byref(a), P, 1 << 60, None) == status
    assert layer.lib.swz_attention_backward(ctypes.byref(a), h, h, h, h, P, 1 << 60, None) == status
    if status != OVERFLOW:
        assert layer.lib.swz_attention_backward_workspace(ctypes.byref(a)) == layer.lib.swz_attention_workspace(ctypes.byref(a)) == status


def test_attention_workspace_refusals():
    many = ctypes.byref(prompt_args(total_k=100000))         # few queries, many keys: cut among workgroups
    need = layer.lib.swz_attention_workspace(many)
    assert need > 0 and layer.lib.swz_attention_workspace(ctypes.byref(prompt_args())) == 0
    assert layer.lib.swz_attention(many, None, need, None) == layer.lib.swz_attention(many, P, need - 1, None) == INVALID
    assert layer.lib.swz_attention(many, P + 8, need, None) == UNSUPPORTED


def test_attention_backward_refusals():
    a, h = ctypes.byref(prompt_args()), heads()
    r = ctypes.byref
    need = layer.lib.swz_attention_backward_workspace(a)
    assert need >= 3 * 2 * 4
    assert layer.lib.swz_attention_backward(a, r(h), r(h), r(h), r(h), P, need - 1, None) == INVALID
    assert layer.lib.swz_attention_backward(a, r(h), r(h), r(h), r(h), None, need, None) == INVALID
    assert layer.lib.swz_attention_backward(a, r(h), r(h), None, r(h), P, need, None) == INVALID
    assert layer.lib.swz_attention_backward(a, r(h), r(h), r(heads(head=1)), r(h), P, need, None) == UNSUPPORTED
    assert layer.lib.swz_attention_backward(a, r(h), r(h), r(h), r(h), P + 4, need, None) == UNSUPPORTED
    assert layer.lib.swz_attention(ctypes.byref(prompt_args(total_q=0)), None, 0, None) == 0


@pytest.mark.parametrize("change,status", [(dict(k_words=None), INVALID), (dict(v_scales=None), INVALID), (dict(pages=0), INVALID), (dict(k_heads=0), INVALID),
                                           (dict(page_tokens=16), UNSUPPORTED), (dict(page_tokens=96), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
                                           (dict(v_words=P + 4), UNSUPPORTED), (dict(pages=1 << 31), OVERFLOW)])
def test_cache_refusals(change, status):
    c, h = ctypes.byref(cache_args(**change)), ctypes.byref(heads())
    for f in (layer.lib.swz_cache4_append, layer.lib.swz_cache4_read):
        assert f(c, h, h, 5, P, P, P, 4, 2, None) == status
    assert layer.lib.swz_cache4_attention_workspace(c, 2, 2, 4, 0) == status
    assert layer.lib.swz_cache4_attention(c, h, h, P, P, 4, 2, 2, 0, 0.1, P, 1 << 40, None) == status


def test_cache_call_refusals():
    c, h, L = ctypes.byref(cache_args()), ctypes.byref(heads()), layer.lib
    for f in (L.swz_cache4_append, L.swz_cache4_read):
        assert f(c, None, h, 5, P, P, P, 4, 2, None) == f(c, h, h, 5, None, P, P, 4, 2, None) == f(c, h, h, -1, P, P, P, 4, 2, None) == INVALID
        assert f(c, h, h, 5, P, P, P, 0, 2, None) == f(c, h, h, 5, P, P, P, 4, 0, None) == INVALID
        assert f(c, h, ctypes.byref(heads(token=4)), 5, P, P, P, 4, 2, None) == f(c, h, h, 5, P + 1, P, P, 4, 2, None) == UNSUPPORTED
        assert f(c, h, h, 1 << 31, P, P, P, 4, 2, None) == OVERFLOW
        assert f(c, h, h, 0, P, P, P, 4, 2, None) == 0
    a = L.swz_cache4_attention
    assert a(c, None, h, P, P, 4, 2, 2, 0, 0.1, P, 1 << 40, None) == a(c, h, h, None, P, 4, 2, 2, 0, 0.1, P, 1 << 40, None) == INVALID
    assert a(c, h, h, P, P, 0, 2, 2, 0, 0.1, P, 1 << 40, None) == a(c, h, h, P, P, 4, 2, 2, -1, 0.1, P, 1 << 40, None) == INVALID
    for scale in (0.0, float("nan"), float("inf")):
        assert a(c, h, h, P, P, 4, 2, 2, 0, scale, P, 1 << 40, None) == INVALID
    wide = 1 << 12                                       # 2^18 tokens: split, so there is a workspace
    need = L.swz_cache4_attention_workspace(c, 1, 2, wide, 0)
    assert need > 0
    assert a(c, h, h, P, P, wide, 1, 2, 0, 0.1, P, need - 1, None) == a(c, h, h, P, P, wide, 1, 2, 0, 0.1, None, need, None) == INVALID
    assert a(c, h, h, P, P, wide, 1, 2, 0, 0.1, P + 4, need, None) == UNSUPPORTED
    assert L.swz_cache4_attention_workspace(ctypes.byref(cache_args(k_heads=2)), 1, 3, wide, 0) == INVALID
    assert L.swz_cache4_attention_workspace(c, 1, 2, 1 << 26, 0) == OVERFLOW


def test_binding_refuses_tensors_off_the_device():
    torch = pytest.importorskip("torch")
    x, cu = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(AssertionError):
        swz.attention(x, x, x, cu)
    with pytest.raises(AssertionError):
        swz.cache4_attention(x, swz.kv_cache4(2, 2, 64, device="cpu"), cu, cu[None])
