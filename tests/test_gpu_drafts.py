"""GPU parity of the entry points of a step with drafted tokens against the fp64 oracle, whose bounds are entry by entry (oracle/drafts_ref.py)."""
import math

import numpy as np
import pytest

from oracle import drafts_ref as dr

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def swz():
    import paper_2508_20258_amd as m
    assert torch.cuda.is_available()
    return m


def f64(t):
    return t.double().cpu().numpy()


def randn(seed, *shape, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16).cuda()


def ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def cu_of(lens):
    return ints(np.concatenate([[0], np.cumsum(lens)]).astype(np.int64).tolist())


def check(got, want, bound, what):
    ok = np.abs(got - want) <= bound
    assert ok.all(), f"{what}: {np.count_nonzero(~ok)} of {ok.size} outside the bound, worst {np.nanmax(np.abs(got - want) / bound)} times it"


def table_of(lens, page, seed=0, spare=0, width=None):
    """Pages of each sequence in a random order (as lists), -1 behind them; and how many pages there are, `spare` of them nobody's."""
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    order = rng.permutation(sum(need) + spare).tolist()
    width = width or max(1, max(need))
    rows, at = [], 0
    for n in need:
        rows.append(order[at:at + n] + [-1] * (width - n))
        at += n
    return rows, max(1, sum(need) + spare)


def angles(rows, half, seed=0):
    a = torch.rand((rows, half), generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * 6.3
    return a.cos().float().cuda(), a.sin().float().cuda()


def filled(swz, pages, heads, dim, page, value=7.0):
    return swz.Cache16(*(torch.full((pages, heads, page, dim), value, dtype=torch.bfloat16, device="cuda") for _ in range(2)))


def same(a, b):
    """Equal bit for bit, NaN included."""
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


# ---------------------------------------------------------------- appending

APPENDS = [   # tokens and positions before of each sequence, query heads, key heads, dims of a head and of the rotation, neighbours, tokens of a page
    ([1], [0], 1, 1, 128, 128, False, 16), ([1], [15], 4, 1, 64, 64, True, 16), ([3, 0, 5], [0, 9, 31], 8, 2, 128, 64, False, 32), ([7, 1, 64], [100, 0, 63], 6, 3, 64, 16, True, 64),
    ([200], [37], 5, 5, 128, 16, True, 128), ([300, 1], [0, 1000], 12, 2, 64, 32, False, 256), ([0, 0, 2], [1, 2, 3], 32, 8, 128, 128, True, 16), ([2] * 70, list(range(70)), 3, 1, 64, 64, False, 16),
]


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("lens,before,q_heads,k_heads,dim,rotary,inter,page", APPENDS)
def test_append(swz, lens, before, q_heads, k_heads, dim, rotary, inter, page, given):
    n = sum(lens)
    ends = [a + m for a, m in zip(before, lens)]
    rows, pages = table_of(ends, page, seed=n, spare=2)
    # one projection's rows, and two tokens behind the last sequence
    x = randn(n, n + 2, (q_heads + 2 * k_heads) * dim)
    q, k, v = (t.view(n + 2, -1, dim) for t in x.split([q_heads * dim, k_heads * dim, k_heads * dim], 1))
    cos, sin = angles(max(ends) + 70, rotary // 2, seed=dim)
    places = [(b, a + i) for b, (a, m) in enumerate(zip(before, lens)) for i in range(m)]
    at = [(p * 7 + 3) % cos.shape[0] for _, p in places] + [0, 0] if given else [p for _, p in places]
    cache = filled(swz, pages, k_heads, dim, page)
    q_out = torch.full((n + 2, q_heads, dim), 5.0, dtype=torch.bfloat16, device="cuda")
    got = swz.cache16_append(cache, k, v, cu_of(lens), ints(before), ints(rows), q=q, cos=cos, sin=sin, positions=ints(at) if given else None, q_out=q_out, interleaved=inter)
    assert got is q_out and (q_out[n:] == 5).all()
    c, s = f64(cos), f64(sin)
    keys, values = f64(cache.k), f64(cache.v)
    xq, xk, xv, zq = f64(q), f64(k), f64(v), f64(q_out)
    untouched = np.ones((pages, page), dtype=bool)
    for t, (b, p) in enumerate(places):
        want, bound = dr.turned(xq[t], c[at[t]], s[at[t]], inter)
        check(zq[t], want, bound, f"query of token {t}")
        where, place = rows[b][p // page], p % page
        want, bound = dr.turned(xk[t], c[at[t]], s[at[t]], inter)
        check(keys[where, :, place], want, bound, f"key of token {t}")
        assert np.array_equal(values[where, :, place], xv[t])
        untouched[where, place] = False
    for x in (keys, values):
        assert (x.transpose(0, 2, 1, 3)[untouched] == 7).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_append_alone(swz, dim):
    """No rotation: the keys as they are.  Outputs in place, heads before tokens: the bits of dense tensors."""
    lens, before = [20, 13], [5, 40]
    rows, pages = table_of([25, 53], 16)
    k, v, q = randn(1, 33, 3, dim), randn(2, 33, 3, dim), randn(3, 33, 6, dim)
    cache = filled(swz, pages, 3, dim, 16)
    assert swz.cache16_append(cache, k, v, cu_of(lens), ints(before), ints(rows)) is None
    places = [(rows[b][p // 16], p % 16) for b, (a, m) in enumerate(zip(before, lens)) for p in range(a, a + m)]
    for t, (where, place) in enumerate(places):
        assert torch.equal(cache.k[where, :, place], k[t]) and torch.equal(cache.v[where, :, place], v[t])
    cos, sin = angles(100, dim // 2)
    call = dict(cos=cos, sin=sin)
    want = swz.cache16_append(cache, k, v, cu_of(lens), ints(before), ints(rows), q=q, **call)
    keys = cache.k.clone()
    swz.cache16_append(cache, k, v, cu_of(lens), ints(before), ints(rows), **call)                     # without queries
    assert torch.equal(cache.k, keys)
    other = q.transpose(0, 1).contiguous().transpose(0, 1)
    got = swz.cache16_append(cache, k.transpose(0, 1).contiguous().transpose(0, 1), v, cu_of(lens), ints(before), ints(rows), q=other, q_out=other, **call)
    assert got is other and torch.equal(got, want) and torch.equal(cache.k, keys)


def test_append_what_is_not_there(swz):
    """Pages that the cache has not, positions past the table, sequences of a negative start, rows that the tables have not."""
    dim, page = 128, 16
    k, v, q = randn(1, 40, 2, dim), randn(2, 40, 2, dim), randn(3, 40, 2, dim)
    cache = filled(swz, 4, 2, dim, page)
    table = ints([[0, -1, 9], [1, 2, 3], [3, 3, 3], [1 << 30, -(1 << 31), 2]])
    # 20 tokens from 10 on (pages 0, -1), 8 from 44 on (page 3, then past the table), 4 from -2 on, 8 from 12 on (no page, twice)
    cos, sin = angles(16, 32)
    at = ints([0, 15, 16, -1, 1 << 30] + [3] * 35)
    got = swz.cache16_append(cache, k, v, ints([0, 20, 28, 32, 40]), ints([10, 44, -2, 12]), table, q=q, cos=cos, sin=sin, positions=at)
    bad = torch.zeros((40, 1, dim), dtype=torch.bool, device="cuda")
    bad[2:5, :, :64] = True
    assert torch.equal(got.isnan(), bad.expand(40, 2, dim)) and torch.equal(got[2:5, :, 64:], q[2:5, :, 64:])
    want = filled(swz, 4, 2, dim, page)
    want.v[0, :, 10:16] = v[:6].transpose(0, 1)
    want.v[3, :, 12:16] = v[20:24].transpose(0, 1)
    assert torch.equal(cache.v, want.v)
    assert cache.k[0, :, 12:15, :64].isnan().all() and not cache.k[0, :, 12:15, 64:].isnan().any() and (cache.k[1:3] == 7).all()
    # positions that follow from a sequence's start, past the tables and past 2^31
    got = swz.cache16_append(cache, k, v, ints([0, 20, 20, 20, 40]), ints([10, 0, 0, (1 << 31) - 5]), table, q=q, cos=cos, sin=sin)
    assert not got[:6].isnan().any() and got[6:, :, :64].isnan().all() and torch.equal(cache.v, want.v)


@pytest.mark.parametrize("inter", [False, True])
def test_append_infinities_stay_with_their_pairs(swz, inter):
    k = randn(1, 3, 1, 64)
    k[0, 0, 5], k[1, 0, 33], k[2, 0, 60] = math.inf, math.nan, -math.inf
    cache = filled(swz, 1, 1, 64, 16)
    cos, sin = angles(8, 20, seed=2)
    cos, sin = cos[:, :16].contiguous(), sin[:, :16].contiguous()
    swz.cache16_append(cache, k, k, cu_of([3]), ints([0]), ints([[0]]), cos=cos, sin=sin, interleaved=inter)
    odd = ~torch.isfinite(cache.k[0, 0, :3])
    want = torch.zeros_like(odd)
    want[0, [4, 5] if inter else [5, 21]] = True
    want[1, 33] = want[2, 60] = True
    assert torch.equal(odd, want) and same(cache.v[0, 0, :3], k[:, 0])


# ---------------------------------------------------------------- attention

def masks_of(lens, branch):
    from paper_2508_20258_amd import draft_tree
    return [draft_tree([max(0, (i - 1) // branch) for i in range(n)])[0] for n in lens]


def check_attention(q, cache, out, nodes, lens, rows, masks=None, scale=None):
    page = cache.k.shape[2]
    group, scale = q.shape[1] // cache.k.shape[1], scale or q.shape[2] ** -0.5
    q, out = f64(q), f64(out)
    first = 0
    for b, (n, length) in enumerate(zip(nodes, lens)):
        length = min(length, len(rows[b]) * page)
        at = torch.arange(length)
        pages = torch.tensor(rows[b], dtype=torch.int64)[at // page] if length else at
        k, v = (f64(x[pages.cuda(), :, (at % page).cuda()]) if length else np.zeros((0, x.shape[1], x.shape[3])) for x in cache)
        seen = dr.looked_at(n, length, None if masks is None else masks[b])
        for h in range(q.shape[1]):
            want, bound = dr.attention(q[first:first + n, h], k[:, h // group], v[:, h // group], scale, seen)
            check(out[first:first + n, h], want, bound, f"head {h} of sequence {b}")
        first += n


ATTENDS = [   # tokens and lengths of each sequence, query heads, key heads, tokens of a page
    ([1], [1], 1, 1, 16), ([1], [64], 4, 1, 16), ([1, 1], [65, 0], 8, 2, 64), ([2], [2], 3, 1, 32), ([5], [300], 2, 2, 16), ([8, 0, 3], [8, 77, 1000], 8, 2, 128), ([33], [40], 1, 1, 16),
    ([64], [64], 2, 1, 64), ([64], [129], 8, 1, 16), ([63, 1, 17], [64, 500, 81], 4, 4, 32), ([31], [31], 5, 1, 16), ([16, 16], [2000, 100], 16, 1, 64),
    ([5, 3], [3, 0], 4, 2, 16), ([1] * 70, [(i * 13) % 97 for i in range(70)], 4, 2, 16), ([(i * 7) % 20 for i in range(130)], [(i * 31) % 150 for i in range(130)], 2, 1, 16),
]


@pytest.mark.parametrize("branch", [0, 1, 3])
@pytest.mark.parametrize("known", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nodes,lens,q_heads,k_heads,page", ATTENDS)
def test_attention(swz, nodes, lens, q_heads, k_heads, page, dim, known, branch):
    """branch 0: no masks.  The longest length known, and unknown under a wide table, when the work is dealt to all of the device; what was there in places that no position names: NaN."""
    width = max(1, -(-max(lens) // page))
    rows, pages = table_of(lens, page, seed=len(nodes), spare=1, width=width if known else width + 4096 // page)
    seed = sum(lens) + dim
    cache = filled(swz, pages, k_heads, dim, page, math.nan)
    for b, n in enumerate(lens):
        for p in range(0, n, page):
            m = min(page, n - p)
            for x, s in zip(cache, (1, 2)):
                x[rows[b][p // page], :, :m] = randn(seed + s + p, k_heads, m, dim)
    q = randn(seed, sum(nodes), q_heads, dim, scale=2.0)
    masks = masks_of(nodes, branch) if branch else None
    tree = ints([m for block in masks for m in block], torch.int64) if branch else None
    args = (q, cache, cu_of(nodes), ints(lens), ints(rows))
    out = swz.cache16_attention(*args, tree=tree, max_length=max(lens) if known else 0)
    check_attention(q, cache, out, nodes, lens, rows, masks)
    assert torch.equal(out, swz.cache16_attention(*args, tree=tree, max_length=max(lens) if known else 0))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nodes,lens,q_heads,k_heads", [
    ([1] * 20 + [0, 3, 2], [700, 1, 0, 64, 65, 256, 257, 300, 30, 511, 513, 90, 800, 12, 128, 129, 640, 33, 1000, 5, 70, 3, 900], 64, 64),
    ([40, 64, 33, 0, 50, 12, 60, 41, 64, 38, 1, 55], [64, 600, 90, 500, 50, 700, 128, 129, 1000, 320, 640, 200], 64, 64),
    ([64, 1, 50, 64, 0, 40, 64, 33, 64, 64], [1100, 900, 70, 128, 300, 40, 700, 64, 129, 66], 128, 64),
    ([64, 20, 64, 31, 64], [300, 1500, 64, 200, 257], 128, 32),
    ([30] * 70, [30 + (i * 53) % 400 for i in range(70)], 32, 16)])
def test_tiles_of_rows_one_after_another(swz, nodes, lens, q_heads, k_heads, dim):
    """Many key heads, so that a workgroup goes from one tile of rows to the next, of one step or many, and from sequence to sequence."""
    page = 16
    rows, pages = table_of(lens, page, width=400)
    cache = filled(swz, pages, k_heads, dim, page, math.nan)
    for b, n in enumerate(lens):
        for p in range(0, n, page):
            for x, s in zip(cache, (1, 2)):
                x[rows[b][p // page], :, :min(page, n - p)] = randn(100 * b + p + s, k_heads, min(page, n - p), dim)
    q = randn(5, sum(nodes), q_heads, dim, scale=2.0)
    masks = masks_of(nodes, 2)
    args = (q, cache, cu_of(nodes), ints(lens), ints(rows))
    for m in (masks, None):
        out = swz.cache16_attention(*args, tree=None if m is None else ints([x for block in m for x in block], torch.int64))
        check_attention(q, cache, out, nodes, lens, rows, m)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nodes,lens", [([100, 65, 1], [100, 300, 70]), ([200], [1000]), ([300], [200])])
def test_pieces_of_prompts(swz, nodes, lens, dim):
    """Blocks of any length without masks; with masks the tokens from the 65th on are looked at by none."""
    rows, pages = table_of(lens, 32)
    cache = swz.Cache16(randn(1, pages, 2, 32, dim), randn(2, pages, 2, 32, dim))
    q = randn(3, sum(nodes), 4, dim, scale=2.0)
    out = swz.cache16_attention(q, cache, cu_of(nodes), ints(lens), ints(rows))
    check_attention(q, cache, out, nodes, lens, rows)
    rng = np.random.default_rng(4)
    masks = [[int(m) for m in rng.integers(-(1 << 63), 1 << 63, n)] for n in nodes]
    out = swz.cache16_attention(q, cache, cu_of(nodes), ints(lens), ints(rows), tree=ints([m for block in masks for m in block], torch.int64))
    check_attention(q, cache, out, nodes, lens, rows, masks)


@pytest.mark.parametrize("max_length", [0, 100])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nodes,q_heads", [([3, 20, 2], 2), ([30, 64, 9], 4)])
def test_masks_of_any_kind(swz, nodes, q_heads, dim, max_length):
    """Rows that look at nothing at all, at tokens after them, at a few."""
    lens = [n for n in nodes]
    lens[1] += 70
    rows, pages = table_of(lens, 16, width=300)
    cache = swz.Cache16(randn(1, pages, 1, 16, dim), randn(2, pages, 1, 16, dim))
    q = randn(3, sum(nodes), q_heads, dim, scale=2.0)
    rng = np.random.default_rng(dim)
    masks = [[0 if i % 3 == 1 else int(rng.integers(-(1 << 63), 1 << 63)) for i in range(n)] for n in nodes]
    out = swz.cache16_attention(q, cache, cu_of(nodes), ints(lens), ints(rows), tree=ints([m for block in masks for m in block], torch.int64), max_length=max_length)
    check_attention(q, cache, out, nodes, lens, rows, masks)
    assert not out[1].any()


@pytest.mark.parametrize("max_length", [0, 100])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("odd", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("q_heads", [2, 8])
def test_what_is_not_finite_stays_with_what_looks_at_it(swz, odd, dim, q_heads, max_length):
    nodes, lens, page = [12, 15], [100, 15], 16
    rows, pages = table_of(lens, page, width=300)
    masks = masks_of(nodes, 2)
    tree = ints([m for block in masks for m in block], torch.int64)
    q = randn(3, sum(nodes), q_heads, dim)
    for keys in (True, False):
        cache = swz.Cache16(randn(1, pages, 1, page, dim), randn(2, pages, 1, page, dim))
        want = swz.cache16_attention(q, cache, cu_of(nodes), ints(lens), ints(rows), tree=tree, max_length=max_length)
        # token 5 of the first block, tokens 4 and 14 of the second
        for b, j in ((0, 5), (1, 4), (1, 14)):
            p = lens[b] - nodes[b] + j
            cache[0 if keys else 1][rows[b][p // page], 0, p % page, 3] = odd
        out = swz.cache16_attention(q, cache, cu_of(nodes), ints(lens), ints(rows), tree=tree, max_length=max_length)
        looks = torch.tensor([bool(m >> 5 & 1) for m in masks[0]] + [bool(m >> 4 & 1 or m >> 14 & 1) for m in masks[1]])
        # what the others see has not changed, but for sums in another order
        assert torch.isfinite(out[~looks]).all() and ((out[~looks].float() - want[~looks].float()).abs() <= 2.0 ** -7 * want[~looks].float().abs() + 2.0 ** -7).all()
        if not keys:
            assert not torch.isfinite(out[looks][..., 3]).any() and torch.isfinite(out[..., 4:]).all()
        elif math.isnan(odd):
            assert out[looks].isnan().all()


@pytest.mark.parametrize("max_length", [0, 64])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_heads", [1, 16])
def test_pages_that_are_not_there(swz, dim, q_heads, max_length):
    """NaN for the sequences that look at them, and for no other; lengths past the table are cut to it, negative ones are 0."""
    nodes, lens, page = [3, 3, 3, 3], [40, 40, 10000, -5], 16
    cache = swz.Cache16(randn(1, 6, 1, page, dim), randn(2, 6, 1, page, dim))
    rows = [[0, -1, 1] + [-1] * 297, [2, 3, 4] + [-1] * 297, [5, 6, 1 << 30] + [0] * 297, [0] * 300]
    q = randn(3, 12, q_heads, dim)
    out = swz.cache16_attention(q, cache, cu_of(nodes), ints(lens), ints(rows), max_length=max_length)
    assert out[:3].isnan().all() and out[6:9].isnan().all() and not out[9:].any()
    check_attention(q[3:6], cache, out[3:6], [3], [40], rows[1:2])
    rows = [r[:1] for r in rows]
    out = swz.cache16_attention(q, cache, cu_of(nodes), ints(lens), ints(rows), max_length=max_length)
    check_attention(q, cache, out, nodes, [16, 16, 16, 0], rows)


@pytest.mark.parametrize("dim", [64, 128])
def test_attention_layouts(swz, dim):
    nodes, lens = [9, 4], [500, 33]
    rows, pages = table_of(lens, 64)
    cache = swz.Cache16(randn(1, pages, 2, 64, dim), randn(2, pages, 2, 64, dim))
    q = randn(3, 15, 6, dim)
    args = (cache, cu_of(nodes), ints(lens), ints(rows))
    want = swz.cache16_attention(q, *args, out=torch.full_like(q, 3.0))
    assert (want[13:] == 3).all()                             # tokens that no sequence owns
    view = randn(4, 6, 15, 2 * dim)[:, :, dim:].transpose(0, 1)
    view.copy_(q)
    out = torch.full((15, 6, 2 * dim), 3.0, dtype=torch.bfloat16, device="cuda")[:, :, :dim]
    got = swz.cache16_attention(view, *args, out=out)
    assert got is out and torch.equal(got, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = swz.cache16_attention(q[:13], *args, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want[:13])
    assert swz.cache16_attention(q[:0], cache, cu_of([0, 0]), ints(lens), ints(rows)).shape == (0, 6, dim)
    with pytest.raises(AssertionError):
        swz.cache16_attention(q, *args, out=q[:, :1].expand(15, 6, dim))
    with pytest.raises(AssertionError):
        swz.cache16_attention(q, *args, tree=torch.zeros(14, dtype=torch.int64, device="cuda"))


@pytest.mark.parametrize("max_length", [0, 64])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_heads,nodes", [(1, [6, 2, 1, 0]), (8, [8, 7, 5, 1]), (16, [20, 40, 9, 8])])
def test_sequences_that_share_pages(swz, dim, q_heads, nodes, max_length):
    """A prompt that several sequences begin with stands in the cache once; one of them has a page of it twice."""
    lens, page = [300, 217, 160, 256], 16
    rows, pages = table_of(lens, page, width=300)
    for r in rows[1:]:
        r[:8] = rows[0][:8]
    rows[2][3] = rows[2][2]
    cache = swz.Cache16(randn(1, pages, 1, page, dim), randn(2, pages, 1, page, dim))
    q = randn(3, sum(nodes), q_heads, dim, scale=2.0)
    masks = masks_of(nodes, 2)
    out = swz.cache16_attention(q, cache, cu_of(nodes), ints(lens), ints(rows), tree=ints([m for block in masks for m in block], torch.int64), max_length=max_length)
    check_attention(q, cache, out, nodes, lens, rows, masks)


@pytest.mark.parametrize("max_length", [0, 64])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_heads", [1, 8, 16])
def test_scores_of_minus_infinity(swz, dim, q_heads, max_length):
    """As if the position were not looked at; nothing but such scores: 0."""
    nodes, lens, page = [9, 12], [400, 130], 16
    rows, pages = table_of(lens, page, width=300)
    cache = swz.Cache16(randn(1, pages, 1, page, dim), randn(2, pages, 1, page, dim))
    q = randn(3, sum(nodes), q_heads, dim)
    q[..., 3] = 1
    gone = [(0, p) for p in range(400) if p % 7 == 0 or 64 <= p < 200 or p < 20] + [(1, p) for p in range(130)]
    for b, p in gone:
        cache.k[rows[b][p // page], 0, p % page, 3] = -math.inf
    out = swz.cache16_attention(q, cache, cu_of(nodes), ints(lens), ints(rows), max_length=max_length)
    assert not out[9:].any()
    # the others' alone: the positions before the block that are left, and a chain of its tokens that misses some
    left = [p for p in range(391) if (0, p) not in gone]
    dense = swz.kv_cache16(40, 1, dim, page)
    places = left + list(range(391, 400))
    for i, p in enumerate(places):
        for x, y in zip(dense, cache):
            x[i // page, 0, i % page] = y[rows[0][p // page], 0, p % page]
    dense.k[:, :, :, 3].clamp_(min=-100)
    masks = [[sum(1 << j for j in range(i + 1) if (0, 391 + j) not in gone) for i in range(9)]]
    check_attention(q[:9], dense, out[:9], [9], [len(places)], [list(range(40))], masks)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scale,size", [(0.02, 1.0), (1.0, 3.0)])
def test_attention_scales(swz, dim, scale, size):
    """Flat weights; and scores whose maximum moves by far more than the kernel leaves unrescaled."""
    nodes, lens = [20, 1], [700, 650]
    rows, pages = table_of(lens, 16)
    cache = swz.Cache16(randn(1, pages, 1, 16, dim, scale=size), randn(2, pages, 1, 16, dim))
    cache.k[rows[0][25]] *= 4
    q = randn(3, 21, 2, dim, scale=size)
    for longest in (0, 64, 700):
        out = swz.cache16_attention(q, cache, cu_of(nodes), ints(lens), ints(rows), scale=scale, max_length=longest)
        check_attention(q, cache, out, nodes, lens, rows, scale=scale)


def test_attention_of_a_long_context(swz):
    """Positions whose keys are past 2^31 bytes from the cache's start, and more pages than a workgroup looks up at once."""
    length, dim, page = 70000, 128, 16
    pages = (1 << 31) // (2 * page * dim * 2) + 4400
    cache = swz.Cache16(*(torch.zeros((pages, 2, page, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    rows = [[pages - 1 - i for i in range(-(-length // page))]]
    for i, x in enumerate(cache):
        x[-4400:] = randn(i, 4400, 2, page, dim)
    q = randn(3, 3, 4, dim, scale=2.0)
    for longest in (0, 64):
        out = swz.cache16_attention(q, cache, cu_of([3]), ints([length]), ints(rows), max_length=longest)
        check_attention(q, cache, out, [3], [length], rows)


# ---------------------------------------------------------------- verification

def probabilities(seed, rows, vocab, half, sharp=2.0):
    x = torch.randn((rows, vocab), generator=torch.Generator().manual_seed(seed)) * sharp
    y = x + torch.randn((rows, vocab), generator=torch.Generator().manual_seed(seed + 1))
    return [t.softmax(1).to(torch.bfloat16 if half else torch.float32).cuda() for t in (x, y)]


def check_verify(got, target, tokens, uniforms, nodes, draft, parents):
    accepted, path, token = (t.tolist() for t in got)
    target, uniforms = f64(target), f64(uniforms)
    draft = None if draft is None else f64(draft)
    tokens, parents = tokens.tolist(), None if parents is None else parents.tolist()
    first = 0
    for b, n in enumerate(nodes):
        part = slice(first, first + n)
        want = dr.verify(target[part], tokens[part], uniforms[part], None if draft is None else draft[part], None if parents is None else parents[part])
        assert (accepted[b], path[part], token[b]) == want, f"sequence {b}"
        first += n


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("branch", [0, 1, 2, 4])
@pytest.mark.parametrize("nodes,vocab", [([1], 1), ([3, 0, 1], 2), ([6] * 20, 37), ([5, 64, 1, 0, 13], 4096), ([8, 9], 4097), ([20, 7, 30], 32003), ([70, 3], 100), ([2, 3], 1100003)])
def test_verify(swz, nodes, vocab, branch, drawn, half):
    """branch 0: a chain without parents."""
    n = sum(nodes)
    target, draft = probabilities(n + vocab, n, vocab, half)
    rng = np.random.default_rng(n)
    parents = [max(0, (i - 1) // max(1, branch)) for m in nodes for i in range(m)]
    first = [sum(nodes[:b]) for b, m in enumerate(nodes) for _ in range(m)]
    rows = draft.float().cpu()
    tokens = []
    for i, (f, p) in enumerate(zip(first, parents)):
        tokens.append(int(rows[f + p].argmax()) if rng.random() < 0.5 else int(torch.multinomial(rows[f + p], 1, generator=torch.Generator().manual_seed(i))) if vocab < 1 << 20 else i)
    tokens, uniforms = ints(tokens), torch.tensor(rng.random(n), dtype=torch.float32, device="cuda")
    parents = ints(parents) if branch else None
    got = swz.verify_drafts(target, tokens, cu_of(nodes), uniforms, draft_probs=draft if drawn else None, parents=parents)
    check_verify(got, target, tokens, uniforms, nodes, draft if drawn else None, parents)


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("seed", range(4))
def test_verify_ties_and_borders(swz, seed, drawn):
    """Probabilities and random numbers in eighths: tests and sums that meet their borders exactly, rows of zeros, drafts that equal the target, children alike."""
    rng = np.random.default_rng(seed)
    nodes, vocab = [int(m) for m in rng.integers(1, 12, 60)], 9
    n = sum(nodes)
    rows = [torch.tensor(rng.multinomial(8, np.full(vocab, 1 / vocab), n) / 8, dtype=torch.float32, device="cuda") for _ in range(2)]
    rows[1][::3] = rows[0][::3]
    rows[0][5::17] = 0
    tokens, uniforms = ints(rng.integers(0, vocab, n).tolist()), torch.tensor(rng.integers(0, 8, n) / 8, dtype=torch.float32, device="cuda")
    parents = ints([int(rng.integers(0, i)) if i else 0 for m in nodes for i in range(m)])
    draft = rows[1] if drawn else None
    for p in (parents, None):
        got = swz.verify_drafts(rows[0], tokens, cu_of(nodes), uniforms, draft_probs=draft, parents=p)
        check_verify(got, rows[0], tokens, uniforms, nodes, draft, p)


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("branch", [0, 3])
def test_verify_odd_inputs(swz, branch, drawn):
    """Tokens outside the vocabulary, parents that are no earlier node, rows that are not finite or negative, random numbers at and past the ends."""
    nodes, vocab = [13, 7, 9, 1, 1, 1, 4], 300
    n = sum(nodes)
    target, draft = probabilities(5, n, vocab, False, sharp=1.0)
    target, draft = target.clone(), draft.clone()
    rng = np.random.default_rng(1)
    tokens = rng.integers(0, vocab, n)
    tokens[[2, 15, 21]] = [-1, vocab, 1 << 30]
    target[0, 7], target[13, 9] = math.nan, math.inf
    target[22:24, ::2] = -1.0
    draft[22:24, 1::3] = -0.5
    target[29] = math.nan
    target[30] = 0
    uniforms = torch.tensor(rng.random(n), dtype=torch.float32)
    uniforms[[0, 13, 20, 31]] = torch.tensor([0.0, 0.5, 1.0, 2.0])
    uniforms[35] = 0.0
    parents = [max(0, (i - 1) // 3) for m in nodes for i in range(m)]
    parents[4], parents[9], parents[16], parents[17] = -1, 9, 12, 1 << 30
    tokens, parents = ints(tokens.tolist()), ints(parents) if branch else None
    got = swz.verify_drafts(target, tokens, cu_of(nodes), uniforms.cuda(), draft_probs=draft if drawn else None, parents=parents)
    check_verify(got, target, tokens, uniforms, nodes, draft if drawn else None, parents)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("u", [0.0, 0.9, 0.999])
def test_verify_siblings_of_one_without_a_probability(swz, u, half):
    """Points, and a failed one whose probability is NaN: no mass is left that a sibling could be tested against, so none passes.  At the root, further down, and where the NaN comes second."""
    vocab, nodes = 5, [3, 6, 5, 4]
    n = sum(nodes)
    target = torch.full((n, vocab), 0.125, dtype=torch.bfloat16 if half else torch.float32)
    target[:, 4] = 0.5
    target[0] = torch.tensor([math.nan, 0.0078125, 0.5, 0.25, 0.0])
    target[3 + 1, 0] = target[9, 1] = math.nan               # of the node that stands; of the second child
    parents = [0, 0, 0, 0, 0, 1, 1, 1, 1, 0, 0, 0, 0, 0, 0, 0, 0, 0]
    tokens = [0, 0, 1, 0, 4, 0, 1, 4, 2, 0, 0, 1, 4, 2, 0, 4, 4, 2]
    uniforms = torch.full((n,), u, dtype=torch.float32)
    uniforms[[0, 3, 9, 14]] = 0.4
    uniforms[4] = 0.0                                        # passes
    uniforms[10] = 0.9                                       # fails
    uniforms[14 + 1] = math.nan                              # no number to test by: fails too
    tokens, parents = ints(tokens), ints(parents)
    got = swz.verify_drafts(target.cuda(), tokens, cu_of(nodes), uniforms.cuda(), parents=parents)
    assert got[0].tolist()[:3] == [0, 1, 0]
    check_verify(got, target, tokens, uniforms, nodes, None, parents)


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("vocab", [300, 9001])
@pytest.mark.parametrize("failing", [1, 31, 32, 62, 63])
def test_verify_many_siblings(swz, failing, vocab, drawn):
    """Nodes of as many children as a block has room for, of which so many fail before one passes, or all do: of the root, and of its child."""
    count = min(failing + 2, 64)
    nodes = [count, count, 64]
    n = sum(nodes)
    target, draft = probabilities(failing + vocab, n, vocab, False)
    draft = (0.7 * target + 0.3 * draft).contiguous()        # much of the target is left for long
    rows = [target.float().cpu(), draft.float().cpu()]
    parents = [0] * count + [0, 0] + [1] * (count - 2) + [0] * 64
    tokens, first = [], 0
    rng = np.random.default_rng(failing)
    for m in nodes:
        for i in range(m):
            p, q = (x[first + parents[first + i]] for x in rows)
            if first == count and i == 1 or first < 2 * count and i == failing + 1:
                tokens.append(int((p / q).argmax()))         # of what is left
            else:
                tokens.append(int((p / q).topk(40 + i, largest=False).indices[-1 - int(rng.integers(0, 20))]))     # of what is not
        first += m
    uniforms = torch.tensor(0.9 + 0.1 * rng.random(n), dtype=torch.float32)
    for at in (failing + 1, count + 1, count + failing + 1):
        if at < 2 * count:
            uniforms[at] = 0.0
    uniforms[[0, count, 2 * count]] = torch.tensor([0.3, 0.5, 0.9])
    tokens, parents, uniforms = ints(tokens), ints(parents), uniforms.cuda()
    got = swz.verify_drafts(target, tokens, cu_of(nodes), uniforms, draft_probs=draft if drawn else None, parents=parents)
    assert int(got[0][1]) >= 1 and int(got[0][2]) == 0 and (failing == 63 or int(got[0][0]) == 1)
    check_verify(got, target, tokens, uniforms, nodes, draft if drawn else None, parents)


@pytest.mark.parametrize("half", [False, True])
def test_verify_layouts(swz, half):
    """Rows apart, starting anywhere; tokens behind the last sequence; no tokens; another stream."""
    nodes, vocab = [4, 3], 1001
    target, draft = probabilities(3, 9, vocab, half)
    tokens, uniforms = ints([5, 17, 900, 3, 8, 8, 1, 2, 3]), torch.rand(9, generator=torch.Generator().manual_seed(1)).cuda()
    tokens[1:4], tokens[5:7] = draft[:3].argmax(1), draft[4:6].argmax(1)
    want = swz.verify_drafts(target, tokens, cu_of(nodes), uniforms, draft_probs=draft)
    check_verify(want, target, tokens, uniforms, nodes, draft, None)
    wide = [torch.full((9, 2 * vocab + 5), 9.0, dtype=t.dtype, device="cuda") for t in (target, draft)]
    views = [w[:, 3:3 + vocab] for w in wide]
    for a, b in zip(views, (target, draft)):
        a.copy_(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = swz.verify_drafts(views[0], tokens, cu_of(nodes), uniforms, draft_probs=views[1], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1][:7], want[1][:7]) and torch.equal(got[2], want[2])
    none = swz.verify_drafts(target[:0], tokens[:0], cu_of([0, 0, 0]), uniforms[:0])
    assert none[0].tolist() == [0, 0, 0] and none[1].shape == (0,) and none[2].tolist() == [-1, -1, -1]
    with pytest.raises(AssertionError):
        swz.verify_drafts(target, tokens, cu_of(nodes), uniforms, draft_probs=draft.double())
    with pytest.raises(AssertionError):
        swz.verify_drafts(target[:1].expand(9, vocab), tokens, cu_of(nodes), uniforms)


# ---------------------------------------------------------------- keeping

@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads", [1, 3, 9, 40])
def test_keep(swz, heads, dim, page):
    nodes, before = [1, 8, 64, 0, 20, 13, 5], [3, 30, 60, 4, 15, 16, 9]
    paths = [[0], [0, 2, 5, 7], [0] + list(range(2, 64)), [], [0, 1, 2, 3, 19], [0], [0, 3]]
    accepted = [0, 3, 62, 0, 4, 0, 1]
    rows, pages = table_of([a + n for a, n in zip(before, nodes)], page, spare=1)
    cache = swz.Cache16(randn(1, pages, heads, page, dim), randn(2, pages, heads, page, dim))
    want = [x.clone() for x in cache]
    for b, path in enumerate(paths):
        for i, node in enumerate(path):
            for x, y in zip(want, cache):
                x[rows[b][(before[b] + i) // page], :, (before[b] + i) % page] = y[rows[b][(before[b] + node) // page], :, (before[b] + node) % page]
    flat = [p for path, n in zip(paths, nodes) for p in (path + [-1] * n)[:n]]
    swz.cache16_keep(cache, cu_of(nodes), ints(before), ints(flat), ints(accepted), ints(rows))
    assert torch.equal(cache.k, want[0]) and torch.equal(cache.v, want[1])


def test_keep_what_is_not_there(swz):
    """Entries that name no token of the block, positions without a page or past the table, counts past the block: left out."""
    page, dim = 16, 64
    cache = swz.Cache16(randn(1, 3, 2, page, dim), randn(2, 3, 2, page, dim))
    want = [x.clone() for x in cache]
    nodes, before = [6, 6, 6, 4], [0, 14, 27, -3]
    path = [0, 6, 3, -2, 5, 1 << 30] + [0, 3, 4, 5, -1, -1] + [0, 2, 4, 5, -1, -1] + [0, 2, 3, -1]
    for x in want:
        x[0, :, 2] = x[0, :, 3]
        x[0, :, 4] = x[0, :, 5]
        x[2, :, 28 - 16] = x[2, :, 29 - 16]
        x[2, :, 29 - 16] = x[2, :, 31 - 16]
    swz.cache16_keep(cache, cu_of(nodes), ints(before), ints(path), ints([100, 3, 3, 2]), ints([[0, 9], [1, -1], [-1, 2], [0, 1]]))
    assert torch.equal(cache.k, want[0]) and torch.equal(cache.v, want[1])


# ---------------------------------------------------------------- all of a step

@pytest.mark.parametrize("branch", [1, 3])
@pytest.mark.parametrize("dim,interleaved", [(64, True), (128, False)])
def test_steps(swz, dim, branch, interleaved):
    """Steps as a server makes them.  After each the cache holds the accepted tokens' keys and values, and attention over it is that over the accepted tokens alone."""
    q_heads, k_heads, page, vocab, count = 6, 2, 16, 64, 10
    sequences, longest = 3, 200
    rows, pages = table_of([longest] * sequences, page)
    table, cache = ints(rows), swz.kv_cache16(pages, k_heads, dim, page)
    cos, sin = angles(longest, dim // 2)
    masks, depths = swz.draft_tree([max(0, (i - 1) // branch) for i in range(count)])
    parents = None if branch == 1 else ints([max(0, (i - 1) // branch) for i in range(count)] * sequences)
    tree, depths = ints(masks * sequences, torch.int64), ints(depths * sequences)
    rng = np.random.default_rng(dim + branch)
    prompts = [20, 1, 33]
    k, v = randn(1, sum(prompts), k_heads, dim), randn(2, sum(prompts), k_heads, dim)
    swz.cache16_append(cache, k, v, cu_of(prompts), ints([0] * sequences), table, cos=cos, sin=sin, interleaved=interleaved)
    held = [[(a, b) for a, b in zip(*(t.split(prompts)[s] for t in (k, v)))] for s in range(sequences)]         # keys and values that stand
    lengths, cu = ints(prompts), cu_of([count] * sequences)
    moved = 0
    for step in range(6):
        n = count * sequences
        q, k, v = randn(10 * step, n, q_heads, dim, scale=2.0), randn(10 * step + 1, n, k_heads, dim), randn(10 * step + 2, n, k_heads, dim)
        positions = lengths.repeat_interleave(count) + depths
        turned = swz.cache16_append(cache, k, v, cu, lengths, table, q=q, cos=cos, sin=sin, positions=positions.to(torch.int32), interleaved=interleaved)
        out = swz.cache16_attention(turned, cache, cu, lengths + count, table, tree=tree)
        target, draft = probabilities(step, n, vocab, step % 2 == 1, sharp=1.5)
        tokens = ints(rng.integers(0, vocab, n).tolist())
        for i in range(n):                                   # likely ones
            if i % count:
                parent = i - 1 if parents is None else i - i % count + int(parents[i])
                tokens[i] = target[parent].float().topk(branch).indices[(i % count - 1) % branch]
        uniforms = torch.tensor(rng.random(n) * 0.6, dtype=torch.float32, device="cuda")
        accepted, path, token = swz.verify_drafts(target, tokens, cu, uniforms, draft_probs=draft if step % 3 == 2 else None, parents=parents)
        check_verify((accepted, path, token), target, tokens, uniforms, [count] * sequences, draft if step % 3 == 2 else None, parents)
        swz.cache16_keep(cache, cu, lengths, path, accepted, table)
        for s in range(sequences):
            way = path[s * count:s * count + int(accepted[s]) + 1].tolist()
            moved += way != list(range(len(way)))
            base = len(held[s])
            held[s] += [(k[s * count + i], v[s * count + i]) for i in way]
            # the accepted tokens' own attention, as a chain without drafts beside it
            dense = swz.kv_cache16(-(-len(held[s]) // page), k_heads, dim, page)
            swz.cache16_append(dense, torch.stack([a for a, _ in held[s]]), torch.stack([b for _, b in held[s]]), cu_of([len(held[s])]), ints([0]),
                               torch.arange(dense.k.shape[0], dtype=torch.int32, device="cuda")[None], cos=cos, sin=sin, interleaved=interleaved)
            for x, y in zip(cache, dense):
                got = x[table[s].long()].transpose(1, 2).flatten(0, 1)[:len(held[s])]
                assert torch.equal(got, y.transpose(1, 2).flatten(0, 1)[:len(held[s])])
            mine = [s * count + i for i in way]
            check_attention(turned[mine], dense, out[mine], [len(way)], [base + len(way)], [list(range(dense.k.shape[0]))])
        lengths = lengths + accepted + 1
        assert lengths.tolist() == [len(h) for h in held]
    assert moved or branch == 1


def test_a_step_in_a_graph(swz):
    """Captured and replayed with other contents in the same tensors, eager work between the replays: the eager results every time; and two graphs that run in turn."""
    q_heads, k_heads, dim, page, vocab, nodes = 8, 2, 128, 16, 5000, [7, 7, 3]
    n = sum(nodes)
    rows, pages = table_of([600] * 3, page)
    table, cu = ints(rows), cu_of(nodes)
    cos, sin = angles(700, dim // 2)
    masks = [m for block in masks_of(nodes, 2) for m in block]
    tree, parents = ints(masks, torch.int64), ints([max(0, (i - 1) // 2) for m in nodes for i in range(m)])

    def inputs(seed):
        target, draft = probabilities(seed, n, vocab, False)
        return dict(q=randn(seed, n, q_heads, dim), k=randn(seed + 1, n, k_heads, dim), v=randn(seed + 2, n, k_heads, dim), target=target, draft=draft,
                    tokens=draft.argmax(1).to(torch.int32)[torch.tensor([max(0, i - 1) for i in range(n)]).cuda()].contiguous(),
                    uniforms=torch.rand(n, generator=torch.Generator().manual_seed(seed)).cuda(), lengths=ints([200 + seed, 17, 590]),
                    cache=swz.Cache16(randn(9, pages, k_heads, page, dim), randn(8, pages, k_heads, page, dim)))

    def step(s):
        q = swz.cache16_append(s["cache"], s["k"], s["v"], cu, s["lengths"], table, q=s["q"], cos=cos, sin=sin)
        out = swz.cache16_attention(q, s["cache"], cu, s["lengths"] + ints_of_nodes, table, tree=tree)
        first = swz.verify_drafts(s["target"], s["tokens"], cu, s["uniforms"], draft_probs=s["draft"], parents=parents)
        second = swz.verify_drafts(s["target"], s["tokens"], cu, s["uniforms"], parents=parents)
        swz.cache16_keep(s["cache"], cu, s["lengths"], first[1], first[0], table)
        return (q, out, *first, *second, *s["cache"])

    ints_of_nodes = ints(nodes)
    states = [inputs(seed) for seed in (1, 2)]
    wants = {seed: [t.clone() for t in step(inputs(seed))] for seed in (1, 2, 3)}
    graphs = []
    for s in states:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(s)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = step(s)
        graphs.append((g, outs))
    for turn in range(6):
        seed = 1 + turn % 3
        for s, (g, outs) in zip(states, graphs):
            for name, value in inputs(seed).items():
                for a, b in zip(s[name], value) if name == "cache" else [(s[name], value)]:
                    a.copy_(b)
            g.replay()
        for _, outs in graphs:
            assert all(torch.equal(a, b) for a, b in zip(outs, wants[seed])), (turn, [torch.equal(a, b) for a, b in zip(outs, wants[seed])])
        step(inputs(seed))
        torch.cuda.synchronize()


def test_steps_on_two_streams_at_once(swz):
    """Two batches with a cache each, every call on a stream of its own, none waiting for the other's: the results of one after the other."""
    q_heads, k_heads, dim, page, vocab, nodes = 8, 2, 64, 32, 20000, [6] * 12
    n, lens = sum(nodes), [100 + 150 * i for i in range(12)]
    rows, pages = table_of([m + 6 for m in lens], page)
    table, cu, before, after = ints(rows), cu_of(nodes), ints(lens), ints([m + 6 for m in lens])
    cos, sin = angles(2000, dim // 2)
    parents = ints([max(0, (i - 1) // 2) for m in nodes for i in range(m)])
    tree = ints([m for block in masks_of(nodes, 2) for m in block], torch.int64)
    tokens = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()

    def state(seed):
        target, draft = probabilities(seed, n, vocab, False)
        return dict(cache=swz.Cache16(randn(seed, pages, k_heads, page, dim), randn(seed + 1, pages, k_heads, page, dim)), k=randn(seed + 2, n, k_heads, dim), v=randn(seed + 3, n, k_heads, dim),
                    q=randn(seed + 4, n, q_heads, dim), target=target, draft=draft, uniforms=torch.rand(n, generator=torch.Generator().manual_seed(seed)).cuda())

    def step(s, stream):
        q = swz.cache16_append(s["cache"], s["k"], s["v"], cu, before, table, q=s["q"], cos=cos, sin=sin, stream=stream)
        out = swz.cache16_attention(q, s["cache"], cu, after, table, tree=tree, stream=stream)
        results = swz.verify_drafts(s["target"], tokens, cu, s["uniforms"], draft_probs=s["draft"], parents=parents, stream=stream)
        swz.cache16_keep(s["cache"], cu, before, results[1], results[0], table, stream=stream)
        return [q, out, *results, *s["cache"]]

    wants = [step(state(seed), None) for seed in (1, 2)]
    states, streams = [[state(seed) for _ in range(5)] for seed in (1, 2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[step(states[i][turn], streams[i]) for i in range(2)] for turn in range(5)]
    torch.cuda.synchronize()
    for turn in got:
        for mine, want in zip(turn, wants):
            assert all(torch.equal(a, b) for a, b in zip(mine, want))


@pytest.mark.parametrize("dim", [64, 128])
def test_a_cache_beyond_32_bits(swz, dim):
    """Pages, and their elements, past 2^32 of the cache's start: the results of a small cache."""
    k_heads, page, nodes, lens = 2, 64, [5, 3], [200, 90]
    rows, pages = table_of([205, 93], page)
    far = (1 << 32) // (k_heads * page * dim) + 7
    small = swz.Cache16(*(randn(i, pages, k_heads, page, dim) for i in range(2)))
    big = swz.Cache16(*(torch.empty((far + pages, k_heads, page, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    k, v, q = randn(3, 8, k_heads, dim), randn(4, 8, k_heads, dim), randn(5, 8, 8, dim)
    cos, sin = angles(300, dim // 2)
    path, accepted = ints([0, 2, 4, -1, -1, 0, 2, -1]), ints([2, 1])
    results, held = [], [x.clone() for x in small]
    for x, y in zip(big, small):
        x[far:] = y
    for cache, first in ((small, 0), (big, far)):
        table = ints([[p + first if p >= 0 else -1 for p in r] for r in rows])
        turned = swz.cache16_append(cache, k, v, cu_of(nodes), ints(lens), table, q=q, cos=cos, sin=sin)
        out = [swz.cache16_attention(turned, cache, cu_of(nodes), ints([a + b for a, b in zip(lens, nodes)]), table, max_length=m) for m in (0, 64)]
        swz.cache16_keep(cache, cu_of(nodes), ints(lens), path, accepted, table)
        results.append([turned, *out, *(x[first:] for x in cache)])
    assert not any(torch.equal(a, b) for a, b in zip(held, small))
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("drawn", [False, True])
def test_probabilities_beyond_32_bits(swz, drawn):
    """Rows that start past 2^32 elements from the first one."""
    vocab, pitch, total = 5000, (1 << 31) - 8, 5
    target, draft = probabilities(7, total, vocab, True)
    wide = torch.empty(pitch * (total - 1) + vocab, dtype=torch.bfloat16, device="cuda").as_strided((total, vocab), (pitch, 1))
    parents = ints([0, 0, 0, 2, 2])
    tokens = ints([0, int(draft[0].argmin()), int(target[0].argmax()), int(target[2].argmin()), int(target[2].argmax())])
    uniforms = torch.tensor([0.7, 0.9, 0.01, 0.99, 0.01], device="cuda")
    call = dict(parents=parents, draft_probs=draft if drawn else None)
    want = swz.verify_drafts(target, tokens, cu_of([total]), uniforms, **call)
    check_verify(want, target, tokens, uniforms, [total], draft if drawn else None, parents)
    wide.copy_(target)
    assert all(torch.equal(a, b) for a, b in zip(swz.verify_drafts(wide, tokens, cu_of([total]), uniforms, **call), want))
    if drawn:
        wide.copy_(draft)
        assert all(torch.equal(a, b) for a, b in zip(swz.verify_drafts(target, tokens, cu_of([total]), uniforms, parents=parents, draft_probs=wide), want))


# ---------------------------------------------------------------- starts of sequences that make no sense

# of 64 tokens: an end beyond them, a start before them, falling and overlapping starts, all that 32 bits hold, and more sequences than are looked at together
SENSELESS = [[0, 1000], [-50, 30], [0, 60, 20, 64], [64, 0], [-(1 << 31), (1 << 31) - 1], [10, 5, 40, -7, 64, (1 << 31) - 1, 0], list(range(100, -40, -2)), [(i * 37) % 90 - 10 for i in range(140)]]


class Fenced:
    """Memory of a call between words that it must leave alone."""
    def __init__(self):
        self.all = []

    def __call__(self, *shape, dtype=torch.bfloat16, value=7):
        n, edge = math.prod(shape), 4096
        whole = torch.full((n + 2 * edge,), value, dtype=dtype, device="cuda")
        self.all.append((whole, edge, n, value))
        return whole[edge:edge + n].view(shape)

    def check(self):
        torch.cuda.synchronize()
        for whole, edge, n, value in self.all:
            assert (whole[:edge] == value).all() and (whole[edge + n:] == value).all()


def owned(cu, total):
    """First token and length of each sequence, cut to the tokens there are."""
    cut = [max(0, min(total, c)) for c in cu]
    return [(a, max(0, b - a)) for a, b in zip(cut, cut[1:])]


@pytest.mark.parametrize("cu", SENSELESS)
@pytest.mark.parametrize("dim", [64, 128])
def test_append_and_keep_stay_inside_the_tensors(swz, cu, dim):
    total, page, heads = 64, 16, 2
    spans, n = owned(cu, total), len(cu) - 1
    fenced = Fenced()
    rows = [[6 * b + j for j in range(6)] for b in range(n)]
    cache = swz.Cache16(*(fenced(6 * n, heads, page, dim) for _ in range(2)))
    k, v, q = randn(1, total, heads, dim), randn(2, total, heads, dim), randn(3, total, 3, dim)
    cos, sin = angles(200, dim // 2)
    q_out = fenced(total, 3, dim)
    before = [(5 * b) % 20 for b in range(n)]
    args = (ints(cu), ints(before), ints(rows))
    swz.cache16_append(cache, k, v, *args, q=q, cos=cos, sin=sin, q_out=q_out)
    fenced.check()
    # a token belongs to the last sequence that starts at it or before, where starts rise; it is written to one place or to none
    mine = torch.zeros(total, dtype=torch.bool)
    for first, length in spans:
        mine[first:first + length] = True
    assert (q_out[~mine.cuda()] == 7).all()
    written = (cache.v != 7).any(-1).any(1).sum()
    assert int(written) <= int(mine.sum())
    if all(a <= b for a, b in zip(cu, cu[1:])):
        want = swz.Cache16(*(torch.full_like(x, 7) for x in cache))
        got = swz.cache16_append(want, k, v, ints([max(0, min(total, c)) for c in cu]), *args[1:], q=q, cos=cos, sin=sin, q_out=torch.full_like(q_out, 7))
        assert torch.equal(got, q_out) and torch.equal(want.k, cache.k) and torch.equal(want.v, cache.v)
    # each sequence's nodes but the second one, in its places: where they overlap, the last sequence's
    path = torch.zeros(total, dtype=torch.int32)
    for first, length in spans:
        path[first:first + length] = torch.tensor([0] + [i + 1 if i + 1 < length else -1 for i in range(1, length)])[:length]
    held = [x.clone() for x in cache]
    accepted = [[0, 5, 1000, -3, (1 << 31) - 1][b % 5] for b in range(n)]
    path = path.tolist()
    swz.cache16_keep(cache, args[0], args[1], ints(path), ints(accepted), args[2])
    fenced.check()
    for b, (first, length) in enumerate(spans):
        moves = [(i, path[first + i]) for i in range(1, min(accepted[b], length - 1) + 1) if path[first + i] >= 0]
        if any(node < i for i, node in moves) or any(y <= x for (_, x), (_, y) in zip(moves, moves[1:])):
            continue                                         # a path that does not rise, of sequences that overlap: any order
        for i, node in moves:
            for x in held:
                x[rows[b][(before[b] + i) // page], :, (before[b] + i) % page] = x[rows[b][(before[b] + node) // page], :, (before[b] + node) % page]
        for x, y in zip(held, cache):
            assert torch.equal(x[rows[b]], y[rows[b]]), b


@pytest.mark.parametrize("cu", SENSELESS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_heads", [1, 4, 8])
@pytest.mark.parametrize("width,max_length", [(5, 0), (300, 0), (300, 64)])
def test_attention_stays_inside_the_tensors(swz, cu, q_heads, dim, width, max_length):
    """Tiles of 32, 64 and 128 rows, alone and dealt; lengths of all kinds, and longer ones than max_length says."""
    from paper_2508_20258_amd import drafts
    total, page, n = 64, 16, len(cu) - 1
    fenced = Fenced()
    lens = [[300, 70, 0, -5, (1 << 31) - 1, 33][b % 6] for b in range(n)]
    rows = [[(7 * b + j) % 40 if j % 11 != 10 else -1 for j in range(width)] for b in range(n)]
    cache = swz.Cache16(randn(1, 40, 1, page, dim), randn(2, 40, 1, page, dim))
    q, out, tree = randn(3, total, q_heads, dim), fenced(total, q_heads, dim), ints([m for block in masks_of([32, 32], 2) for m in block], torch.int64)
    c = drafts._cache(cache)
    tensors = ints(cu), ints(lens), ints(rows)
    for mask in (None, tree):
        a = drafts._DraftAttentionArgs(drafts._heads(q), drafts._heads(out), *(t.data_ptr() for t in tensors), None if mask is None else mask.data_ptr(), total, n, width, q_heads, max_length, 0.1)
        need = drafts.lib.swz_cache16_attention_workspace(drafts.ctypes.byref(c), drafts.ctypes.byref(a))
        assert need >= 0
        # what a part's place would be that nobody wrote: any numbers, other ones each time
        for value in (0, 1, 255):
            work = fenced(max(need, 16), dtype=torch.uint8, value=value)
            out.fill_(7)
            assert drafts.lib.swz_cache16_attention(drafts.ctypes.byref(c), drafts.ctypes.byref(a), work.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
            fenced.check()
        mine = torch.zeros(total, dtype=torch.bool)
        for first, length in owned(cu, total):
            mine[first:first + length] = True
        assert (out[~mine.cuda()] == 7).all()
        if all(a <= b for a, b in zip(cu, cu[1:])):
            cut = ints([max(0, min(total, x)) for x in cu])
            want = swz.cache16_attention(q, cache, cut, *tensors[1:], tree=mask, max_length=max_length, scale=0.1, out=torch.full_like(out, 7))
            assert same(out, want)


@pytest.mark.parametrize("cu", SENSELESS)
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("branch", [0, 2])
def test_verification_stays_inside_the_tensors(swz, cu, branch, drawn):
    from paper_2508_20258_amd import drafts
    total, vocab, n = 64, 5000, len(cu) - 1
    fenced = Fenced()
    target, draft = probabilities(1, total, vocab, False)
    tokens, uniforms = ints([int(t) for t in target.argmax(1).roll(1)]), torch.rand(total, generator=torch.Generator().manual_seed(1)).cuda() * 0.5
    parents = ints([max(0, (i % 30 - 1) // 2) for i in range(total)]) if branch else None
    accepted, path, token = fenced(n, dtype=torch.int32), fenced(total, dtype=torch.int32), fenced(n, dtype=torch.int32)
    starts = ints(cu)
    a = drafts._VerifyArgs(target.data_ptr(), draft.data_ptr() if drawn else None, vocab, vocab, vocab, total, tokens.data_ptr(), None if parents is None else parents.data_ptr(), starts.data_ptr(),
                           uniforms.data_ptr(), accepted.data_ptr(), path.data_ptr(), token.data_ptr(), n, 4)
    need = drafts.lib.swz_verify_drafts_workspace(drafts.ctypes.byref(a))
    work = fenced(need, dtype=torch.uint8, value=255)
    assert drafts.lib.swz_verify_drafts(drafts.ctypes.byref(a), work.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
    fenced.check()
    # each sequence's own, whatever the others; the path where no other one has its places
    target, draft, spans = f64(target), f64(draft) if drawn else None, owned(cu, total)
    many, path = np.zeros(total, dtype=int), path.tolist()
    for first, length in spans:
        many[first:first + length] += 1
    for b, (first, length) in enumerate(spans):
        part = slice(first, first + length)
        want = dr.verify(target[part], tokens[part].tolist(), f64(uniforms[part]), None if draft is None else draft[part], None if parents is None else parents[part].tolist())
        assert (int(accepted[b]), int(token[b])) == (want[0], want[2]), b
        assert all(p == w for p, w, m in zip(path[part], want[1], many[part]) if m == 1), b
    assert all(p == 7 for p, m in zip(path, many) if m == 0)
