"""What the attention entry points say at the ends of their ranges, before anything is launched or written.  No GPU: pointers that are never used."""
import ctypes

import pytest

from paper_2508_20258_amd import attention_layer as layer

P = 0x1000
OK, INVALID, OVERFLOW = 0, -1, -3


def heads(token=256, head=128):
    return layer._Heads(P, token, head)


def prompt_args(**change):
    a = dict(q=heads(), k=heads(), v=heads(), out=heads(), lse=P, cu_q=P, cu_k=P, total_q=3, total_k=3, sequences=1, q_heads=2, k_heads=1, head_dim=128, causal=1, scale=0.1)
    a.update(change)
    return layer._AttentionArgs(*(a[n] for n, _ in layer._AttentionArgs._fields_))


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_no_launch_where_a_later_one_is_too_large(head_dim, causal):
    # two million sequences of about 1070 keys: cut in two, which 12 million workgroups do, and joined for each of 12 heads by twice as many of as many threads
    a = prompt_args(total_q=100, total_k=(1 << 31) - 5000, sequences=2000000, q_heads=12, k_heads=3, head_dim=head_dim, causal=causal)
    need = layer.lib.swz_attention_workspace(ctypes.byref(a))
    assert need > 0
    assert layer.lib.swz_attention(ctypes.byref(a), P, need, None) == OVERFLOW


@pytest.mark.parametrize("head_dim", [64, 128])
def test_no_workspace_where_none_is_needed(head_dim):
    a, h = ctypes.byref(prompt_args(total_q=0, total_k=0, head_dim=head_dim)), ctypes.byref(heads())
    assert layer.lib.swz_attention_workspace(a) == layer.lib.swz_attention_backward_workspace(a) == 0
    assert layer.lib.swz_attention(a, None, 0, None) == layer.lib.swz_attention_backward(a, h, h, h, h, None, 0, None) == OK
    a = ctypes.byref(prompt_args(head_dim=head_dim))
    need = layer.lib.swz_attention_backward_workspace(a)
    assert need > 0 and layer.lib.swz_attention_backward(a, h, h, h, h, None, need, None) == INVALID


# Tiles and steps reach past the last token by less than 4096, in 32-bit numbers: beyond that they would wrap, and a loop over them would not end.
MOST = (1 << 31) - 4096


@pytest.mark.parametrize("head_dim", [64, 128])
def test_tokens_whose_tiles_would_pass_32_bits(head_dim):
    lib, r = layer.lib, ctypes.byref
    for which in ("total_q", "total_k"):
        h = r(heads())
        for tokens in (MOST + 1, (1 << 31) - 1):
            a = prompt_args(head_dim=head_dim, **{which: tokens})
            assert lib.swz_attention_workspace(r(a)) == lib.swz_attention_backward_workspace(r(a)) == OVERFLOW
            assert lib.swz_attention(r(a), P, 1 << 60, None) == lib.swz_attention_backward(r(a), h, h, h, h, P, 1 << 60, None) == OVERFLOW
        a = prompt_args(head_dim=head_dim, **{which: MOST})
        assert lib.swz_attention_workspace(r(a)) >= 0 and lib.swz_attention_backward_workspace(r(a)) > 0


@pytest.mark.parametrize("page", [32, 64, 1024])
def test_tables_whose_steps_would_pass_32_bits(page):
    c, h, lib = ctypes.byref(layer._Cache4(P, P, P, P, 4, page, 1, 128)), ctypes.byref(heads()), layer.lib
    for width in (MOST // page + 1, (1 << 31) // page - 1):
        assert lib.swz_cache4_attention_workspace(c, 1, 2, width, 0) == lib.swz_cache4_attention_workspace(c, 1, 2, width, 100) == OVERFLOW
        assert lib.swz_cache4_attention(c, h, h, P, P, width, 1, 2, 0, 0.1, P, 1 << 60, None) == OVERFLOW
    assert lib.swz_cache4_attention_workspace(c, 1, 2, MOST // page, 0) > 0
