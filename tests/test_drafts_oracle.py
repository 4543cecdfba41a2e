"""The oracle of a step with drafted tokens against closed forms and distributions, and the host side of its entry points: exports, refusals, masks of trees.  No GPU: pointers that are never used."""
import ctypes
import itertools
import os
import re

import numpy as np
import pytest

import paper_2508_20258_amd as swz
from oracle import attention_ref as ar
from oracle import drafts_ref as dr
from paper_2508_20258_amd import attention_layer as layer, drafts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000
OK, INVALID, UNSUPPORTED, OVERFLOW = 0, -1, -2, -3
lib, ref = drafts.lib, ctypes.byref


def test_library_exports_every_declared_entry_point():
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "swz_drafts.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(swz_[a-z0-9_]+)\s*\(", header))
    assert declared == set(drafts.EXPORTS)
    raw = ctypes.CDLL(swz.binding.LIB_PATH)
    for name in declared:
        assert hasattr(raw, name), name


# ---------------------------------------------------------------- the oracle

@pytest.mark.parametrize("n,length", [(1, 1), (3, 3), (3, 7), (5, 2), (2, 0)])
def test_a_chain_is_causal_attention(n, length):
    rng = np.random.default_rng(n * 10 + length)
    q, k, v = (rng.normal(size=(m, 4)) for m in (n, length, length))
    want, _, _, _ = ar.attention(q, k, v, 0.5, True)
    got, _ = dr.attention(q, k, v, 0.5, dr.looked_at(n, length))
    assert np.allclose(got, want, atol=1e-12)
    masks, _ = drafts.draft_tree([0] + list(range(n - 1)))
    assert np.array_equal(dr.looked_at(n, length), dr.looked_at(n, length, masks))


def test_trees():
    masks, depths = drafts.draft_tree([0, 0, 0, 1, 3, 2])
    assert masks == [0b1, 0b11, 0b101, 0b1011, 0b11011, 0b100101] and depths == [0, 1, 1, 2, 3, 2]
    masks, depths = drafts.draft_tree([0] + list(range(63)))
    assert masks[62] == (1 << 63) - 1 and masks[63] == -1 and depths[63] == 63
    assert drafts.draft_tree([]) == ([], [])
    for bad in ([0, 1], [0, 0, 2], [0, -1], [0] * 65):
        with pytest.raises(AssertionError):
            drafts.draft_tree(bad)


def emitted(target, draft, tree, first_child, grid):
    """Distribution of the first token that a step emits, over all draws of the children and a grid of random numbers."""
    vocab, n = target.shape[1], len(tree)
    got = np.zeros(vocab)
    for children in itertools.product(range(vocab), repeat=n - 1) if draft is not None else [first_child]:
        weight = np.prod([draft[0, x] for x in children]) if draft is not None else 1.0
        us = (np.arange(grid) + 0.5) / grid
        for u in itertools.product(us, repeat=n):
            accepted, path, token = dr.verify(target[:n], [0, *children], u, draft, tree)
            got[children[path[1] - 1] if accepted else token] += weight / grid ** n
    return got


@pytest.mark.parametrize("children", [1, 2])
def test_what_is_emitted_has_the_targets_distribution_drawn(children):
    # probabilities whose borders are on the grid's lines, or near enough: within the grid's step a number and test
    p, q = np.array([[0.5, 0.25, 0.25]] * 3), np.array([[0.25, 0.25, 0.5]] * 3)
    got = emitted(p, q, [0] + [0] * children, None, 8)
    assert np.abs(got - p[0]).max() <= 1e-12 if children == 1 else np.abs(got - p[0]).max() < 0.07


@pytest.mark.parametrize("children", [1, 2])
def test_what_is_left_over_is_divided_by_its_sum(children):
    """Two tokens are left over, by unequal parts, one of which the draft draws more often than it is left before the division and less often than after it.  All borders (1/4, 2/3, 1/6) are lines of the grid, so
    that each sum of its cells is the probability, but for one rounding an addition."""
    p, q = np.array([[2, 5, 9]] * 3) / 16, np.array([[8, 4, 4]] * 3) / 16
    got = emitted(p, q, [0] + [0] * children, None, 12)
    assert np.abs(got - p[0]).max() <= 2 * 2.0 ** -53 * 3 ** children * 12 ** (children + 1)


@pytest.mark.parametrize("first", [(0,), (2, 0), (1, 1), (0, 1, 2)])
def test_what_is_emitted_has_the_targets_distribution_points(first):
    p = np.array([[0.5, 0.25, 0.25]] * 4)
    got = emitted(p, None, [0] + [0] * len(first), first, 4 if len(first) == 3 else 12)
    assert np.abs(got - p[0]).max() < 0.07


def test_verify_closed_forms():
    one = np.eye(4)
    # a greedy target: what it would say stands, and then its own word
    assert dr.verify(one[[1, 2, 3]], [0, 1, 2], [0.3, 0.9, 0.9]) == (2, [0, 1, 2], 3)
    assert dr.verify(one[[1, 2, 3]], [0, 1, 3], [0.3, 0.9, 0.9]) == (1, [0, 1, -1], 2)
    # the second child of the root, and its child
    assert dr.verify(one[[2, 0, 3, 1]], [0, 1, 2, 3], [0.0, 0.5, 0.5, 0.5], None, [0, 0, 0, 2]) == (2, [0, 2, 3, -1], 1)
    # no row to draw from
    assert dr.verify(np.zeros((1, 4)), [0], [0.5]) == (0, [0], -1) and dr.verify(np.full((1, 4), np.nan), [0], [0.5])[2] == -1
    # the draft was sure of what the target excludes: the rest, in proportion
    p, q = np.array([[0.0, 0.25, 0.75, 0.0]] * 2), np.array([[1.0, 0.0, 0.0, 0.0]] * 2)
    assert dr.verify(p, [9, 0], [0.24, 0.5], q) == (0, [0, -1], 1) and dr.verify(p, [9, 0], [0.25, 0.5], q) == (0, [0, -1], 2)
    # a draft that left nothing over: the target itself
    assert dr.verify(p, [9, 0], [0.3, 0.5], p) == (0, [0, -1], 2)


def test_no_child_passes_by_a_mass_that_is_no_number():
    p = np.array([[np.nan, 0.01, 0.5, 0.49]] * 3)
    # its probability is none, so what is left of the mass is none; the new token is drawn from the rest of the row
    assert dr.verify(p, [9, 0, 1], [0.3, 0.9, 0.999], None, [0, 0, 0]) == (0, [0, -1, -1], 2)
    assert dr.verify(p, [9, 0, 1], [0.6, 0.9, 0.0], None, [0, 0, 0]) == (0, [0, -1, -1], 3)


# ---------------------------------------------------------------- refusals

def heads(token=256, head=128, at=P):
    return layer._Heads(at, token, head)


def cache(**change):
    return drafts._Cache16(**{**dict(k=P, v=P, pages=4, page_tokens=16, k_heads=2, head_dim=128), **change})


BAD_CACHES = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(pages=0), INVALID), (dict(k_heads=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
              (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED), (dict(page_tokens=0), UNSUPPORTED), (dict(k=P + 8), UNSUPPORTED), (dict(pages=1 << 31), OVERFLOW),
              (dict(k_heads=1 << 17), OVERFLOW)]


def append_args(**change):
    a = dict(q=heads(), k=heads(), v=heads(), q_out=heads(), cos=P, sin=P, positions=P, cu=P, before=P, block_table=P, tokens=3, table_rows=8, sequences=1, table_width=2, q_heads=4,
             rotary_dim=128, interleaved=0)
    return drafts._AppendArgs(**{**a, **change})


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches_that_are_refused(change, status):
    c = ref(cache(**change))
    assert lib.swz_cache16_append(c, ref(append_args()), None) == status
    assert lib.swz_cache16_attention_workspace(c, ref(attention_args())) == lib.swz_cache16_attention(c, ref(attention_args()), P, 1 << 40, None) == status
    assert lib.swz_cache16_keep(c, P, P, P, P, 3, P, 2, 1, None) == status


@pytest.mark.parametrize("change,status", [
    (dict(cu=None), INVALID), (dict(before=None), INVALID), (dict(block_table=None), INVALID), (dict(tokens=-1), INVALID), (dict(sequences=0), INVALID), (dict(table_width=0), INVALID),
    (dict(sin=None), INVALID), (dict(cos=None), INVALID), (dict(cos=None, sin=None), INVALID), (dict(q_heads=0), INVALID), (dict(table_rows=-1), INVALID), (dict(k=heads(at=None)), INVALID),
    (dict(q_out=heads(at=None)), INVALID), (dict(k=heads(token=-8)), INVALID), (dict(k=heads(token=100)), UNSUPPORTED), (dict(v=heads(head=4)), UNSUPPORTED), (dict(q=heads(at=P + 8)), UNSUPPORTED),
    (dict(rotary_dim=8), UNSUPPORTED), (dict(rotary_dim=144), UNSUPPORTED), (dict(rotary_dim=24), UNSUPPORTED), (dict(cos=P + 4), UNSUPPORTED), (dict(positions=P + 2), UNSUPPORTED),
    (dict(before=P + 2), UNSUPPORTED), (dict(cu=P + 1), UNSUPPORTED), (dict(tokens=1 << 31), OVERFLOW), (dict(q_heads=1 << 17), OVERFLOW), (dict(tokens=0), OK)])
def test_append_refuses(change, status):
    assert lib.swz_cache16_append(ref(cache()), ref(append_args(**change)), None) == status


def attention_args(**change):
    a = dict(q=heads(), out=heads(), cu=P, lengths=P, block_table=P, tree=P, tokens=3, sequences=1, table_width=2, q_heads=4, max_length=0, scale=0.1)
    return drafts._DraftAttentionArgs(**{**a, **change})


@pytest.mark.parametrize("change,status", [
    (dict(cu=None), INVALID), (dict(lengths=None), INVALID), (dict(block_table=None), INVALID), (dict(tokens=-1), INVALID), (dict(sequences=0), INVALID), (dict(table_width=0), INVALID),
    (dict(q_heads=3), INVALID), (dict(q_heads=0), INVALID), (dict(max_length=-1), INVALID), (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(tree=P + 4), UNSUPPORTED), (dict(lengths=P + 2), UNSUPPORTED), (dict(tokens=(1 << 31) - 4095), OVERFLOW), (dict(tokens=1 << 30), OVERFLOW), (dict(table_width=1 << 27), OVERFLOW),
    (dict(q_heads=1 << 17), OVERFLOW)])
def test_attention_refuses(change, status):
    a = ref(attention_args(**change))
    assert lib.swz_cache16_attention_workspace(ref(cache()), a) == lib.swz_cache16_attention(ref(cache()), a, P, 1 << 40, None) == status


def test_attention_refuses_heads_and_workspaces():
    for change, status in ((dict(q=heads(at=None)), INVALID), (dict(out=heads(token=100)), UNSUPPORTED), (dict(tokens=0), OK)):
        assert lib.swz_cache16_attention(ref(cache()), ref(attention_args(**change)), P, 1 << 40, None) == status
    a = ref(attention_args(table_width=4096))
    need = lib.swz_cache16_attention_workspace(ref(cache()), a)
    assert need > 0
    for work, size in ((None, need), (P, need - 1), (P, 0)):
        assert lib.swz_cache16_attention(ref(cache()), a, work, size, None) == INVALID
    assert lib.swz_cache16_attention(ref(cache()), a, P + 8, need, None) == UNSUPPORTED


@pytest.mark.parametrize("head_dim", [64, 128])
def test_steps_of_all_rows_fit_32_bits(head_dim):
    c = ref(cache(head_dim=head_dim))
    # 2^21 tokens of 2 query heads of a key head (each sequence one) over tables of 2^20 positions
    big = dict(tokens=1 << 21, sequences=1 << 21, table_width=1 << 16)
    assert lib.swz_cache16_attention_workspace(c, ref(attention_args(**big))) == lib.swz_cache16_attention(c, ref(attention_args(**big)), P, 1 << 60, None) == OVERFLOW
    assert lib.swz_cache16_attention_workspace(c, ref(attention_args(**{**big, "table_width": 16}))) >= 0


def verify_args(**change):
    a = dict(target=P, draft=P, target_pitch=100, draft_pitch=100, vocab=100, total=5, tokens=P, parents=P, cu=P, uniforms=P, accepted=P, path=P, token=P, sequences=2, elem_bytes=4)
    return drafts._VerifyArgs(**{**a, **change})


@pytest.mark.parametrize("change,status", [(dict([(name, None)]), INVALID) for name in ("target", "tokens", "cu", "uniforms", "accepted", "path", "token")] + [
    (dict(vocab=0), INVALID), (dict(total=-1), INVALID), (dict(sequences=0), INVALID), (dict(target_pitch=99), INVALID), (dict(draft_pitch=99), INVALID), (dict(elem_bytes=1), UNSUPPORTED),
    (dict(elem_bytes=8), UNSUPPORTED), (dict(target=P + 2), UNSUPPORTED), (dict(draft=P + 1, elem_bytes=2), UNSUPPORTED), (dict(parents=P + 2), UNSUPPORTED), (dict(tokens=P + 2), UNSUPPORTED),
    (dict(vocab=1 << 30, target_pitch=1 << 30, draft=None), OVERFLOW), (dict(total=1 << 31), OVERFLOW), (dict(target_pitch=1 << 31), OVERFLOW), (dict(sequences=1 << 22), OVERFLOW)])
def test_verify_refuses(change, status):
    a = ref(verify_args(**change))
    assert lib.swz_verify_drafts_workspace(a) == lib.swz_verify_drafts(a, P, 1 << 40, None) == status


def test_verify_refuses_workspaces():
    a = ref(verify_args())
    need = lib.swz_verify_drafts_workspace(a)
    assert need > 0
    assert lib.swz_verify_drafts(a, None, need, None) == lib.swz_verify_drafts(a, P, need - 1, None) == INVALID
    assert lib.swz_verify_drafts(a, P + 8, need, None) == UNSUPPORTED
    assert lib.swz_verify_drafts(ref(verify_args(draft=None, draft_pitch=0)), P, 0, None) == INVALID      # (a pitch without rows is not read)


@pytest.mark.parametrize("change,status", [(dict(cu=None), INVALID), (dict(before=None), INVALID), (dict(path=None), INVALID), (dict(accepted=None), INVALID), (dict(table=None), INVALID),
                                           (dict(tokens=-1), INVALID), (dict(width=0), INVALID), (dict(sequences=0), INVALID), (dict(path=P + 2), UNSUPPORTED), (dict(cu=P + 2), UNSUPPORTED),
                                           (dict(tokens=(1 << 31) - 4095), OVERFLOW), (dict(tokens=0), OK)])
def test_keep_refuses(change, status):
    a = {**dict(cu=P, before=P, path=P, accepted=P, tokens=3, table=P, width=2, sequences=1), **change}
    assert lib.swz_cache16_keep(ref(cache()), a["cu"], a["before"], a["path"], a["accepted"], a["tokens"], a["table"], a["width"], a["sequences"], None) == status


MOST = (1 << 31) - 4096


@pytest.mark.parametrize("page,width", [(16, (1 << 27) + 1), (64, (1 << 25) + 1), (1 << 16, 1 << 15), (1 << 30, 2), (1 << 30, (1 << 31) - 1), (4096, MOST // 4096 + 1)])
def test_tables_of_positions_beyond_32_bits(page, width):
    """Positions are 32-bit numbers on the device: a table that has more of them could be given a start (which the host does not see) from which they would be negative."""
    c = ref(cache(page_tokens=page))
    assert lib.swz_cache16_append(c, ref(append_args(table_width=width)), None) == OVERFLOW
    assert lib.swz_cache16_append(c, ref(append_args(table_width=width, cos=None, sin=None, positions=None, q=heads(at=None))), None) == OVERFLOW
    assert lib.swz_cache16_keep(c, P, P, P, P, 3, P, width, 1, None) == OVERFLOW
    a = ref(attention_args(table_width=width))
    assert lib.swz_cache16_attention_workspace(c, a) == lib.swz_cache16_attention(c, a, P, 1 << 60, None) == OVERFLOW
    # nothing to do
    assert lib.swz_cache16_append(c, ref(append_args(table_width=width, tokens=0)), None) == lib.swz_cache16_keep(c, P, P, P, P, 0, P, width, 1, None) == OK


@pytest.mark.parametrize("page", [16, 4096])
def test_tables_as_wide_as_32_bits_allow(page):
    """(What comes after the checks: no device, no launch.)"""
    widest = MOST // page
    assert widest * page == MOST
    c = ref(cache(page_tokens=page))
    assert lib.swz_cache16_append(c, ref(append_args(table_width=widest, k=heads(at=None))), None) == INVALID
    assert lib.swz_cache16_attention_workspace(c, ref(attention_args(table_width=widest, max_length=64))) >= 0
    assert lib.swz_cache16_keep(c, P, P, P + 2, P, 3, P, widest, 1, None) == UNSUPPORTED
