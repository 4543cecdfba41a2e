"""GPU parity of the attention entry points against the fp64 oracle, whose bounds are entry by entry (oracle/attention_ref.py)."""
import numpy as np
import pytest

from oracle import attention_ref as ar

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


def cu_of(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def check(got, want, bound, what):
    err = np.abs(got - want)
    ok = err <= bound
    assert ok.all(), f"{what}: {np.count_nonzero(~ok)} of {ok.size} outside the bound, worst {np.max(err / bound)} times it"


def sequences(q_lens, k_lens):
    q0 = k0 = 0
    for nq, nk in zip(q_lens, k_lens):
        yield slice(q0, q0 + nq), slice(k0, k0 + nk)
        q0, k0 = q0 + nq, k0 + nk


def check_forward(q, k, v, out, lse, q_lens, k_lens, causal, scale):
    group = q.shape[1] // k.shape[1]
    q, k, v, out, lse = f64(q), f64(k), f64(v), f64(out), f64(lse)
    for rows, keys in sequences(q_lens, k_lens):
        for h in range(q.shape[1]):
            want, l, _, bound = ar.attention(q[rows, h], k[keys, h // group], v[keys, h // group], scale, causal)
            check(out[rows, h], want, bound, f"out of head {h}, {rows}")
            got = lse[h, rows]
            assert np.array_equal(np.isneginf(got), np.isneginf(l))
            some = np.isfinite(l)
            assert (np.abs(got - l)[some] <= 2e-5 * (1 + np.abs(l[some]))).all()


def check_backward(q, k, v, dout, grads, q_lens, k_lens, causal, scale):
    group = q.shape[1] // k.shape[1]
    q, k, v, dout = f64(q), f64(k), f64(v), f64(dout)
    dq, dk, dv = (f64(g) for g in grads)
    for rows, keys in sequences(q_lens, k_lens):
        for kh in range(k.shape[1]):
            sums, bounds = [0.0, 0.0], [0.0, 0.0]
            for h in range(kh * group, (kh + 1) * group):
                want, bound = ar.attention_backward(q[rows, h], k[keys, kh], v[keys, kh], scale, causal, dout[rows, h])
                check(dq[rows, h], want[0], bound[0], f"dq of head {h}, {rows}")
                sums = [s + w for s, w in zip(sums, want[1:])]
                bounds = [s + b for s, b in zip(bounds, bound[1:])]
            check(dk[keys, kh], sums[0], bounds[0], f"dk of head {kh}, {keys}")
            check(dv[keys, kh], sums[1], bounds[1], f"dv of head {kh}, {keys}")


PROMPTS = [
    # lengths of queries, of keys (None: the same), query heads, key heads
    ([1], None, 1, 1), ([2], None, 3, 1), ([31], None, 2, 2), ([32], None, 1, 1), ([33], None, 4, 2), ([63, 64, 65], None, 2, 1), ([127], None, 1, 1), ([129], None, 2, 1),
    ([257], None, 1, 1), ([300, 0, 1, 70], None, 8, 2), ([0, 5], None, 1, 1),
    ([5], [200], 2, 1), ([64], [65], 1, 1), ([130], [300], 2, 2), ([1], [129], 4, 1),                     # the next piece of a prompt
    ([3], [2100], 2, 1), ([70, 1, 0], [1500, 1600, 900], 2, 2),                                         # few queries and many keys: cut among workgroups
    ([40], [7], 2, 1), ([200, 3], [70, 0], 1, 1), ([70], [1], 3, 1),                                     # rows that look at nothing
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_lens,k_lens,q_heads,k_heads", PROMPTS)
def test_attention_and_gradient(swz, q_lens, k_lens, q_heads, k_heads, dim, causal):
    k_lens = k_lens or q_lens
    seed, nq, nk = sum(q_lens) * 7 + dim, sum(q_lens), sum(k_lens)
    q, k, v, dout = randn(seed, nq, q_heads, dim, scale=2.0), randn(seed + 1, nk, k_heads, dim), randn(seed + 2, nk, k_heads, dim), randn(seed + 3, nq, q_heads, dim)
    cu_q, cu_k = cu_of(q_lens), cu_of(k_lens)
    out, lse = swz.attention(q, k, v, cu_q, cu_k, causal=causal)
    check_forward(q, k, v, out, lse, q_lens, k_lens, causal, dim ** -0.5)
    grads = swz.attention_backward(dout, q, k, v, out, lse, cu_q, cu_k, causal=causal)
    check_backward(q, k, v, dout, grads, q_lens, k_lens, causal, dim ** -0.5)
    again = (*swz.attention(q, k, v, cu_q, cu_k, causal=causal), *swz.attention_backward(dout, q, k, v, out, lse, cu_q, cu_k, causal=causal))
    assert all(torch.equal(a, b) for a, b in zip(again, (out, lse, *grads)))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scale,size", [(0.02, 1.0), (1.0, 3.0)])
def test_attention_scales(swz, dim, scale, size):
    # flat weights; and scores whose maximum moves by far more than the kernel leaves unrescaled
    q, k, v, dout = randn(1, 150, 2, dim, scale=size), randn(2, 150, 1, dim, scale=size), randn(3, 150, 1, dim), randn(4, 150, 2, dim)
    k[100:] *= 4
    cu = cu_of([150])
    out, lse = swz.attention(q, k, v, cu, scale=scale)
    check_forward(q, k, v, out, lse, [150], [150], True, scale)
    if scale < 1:
        check_backward(q, k, v, dout, swz.attention_backward(dout, q, k, v, out, lse, cu, scale=scale), [150], [150], True, scale)


@pytest.mark.parametrize("dim", [64, 128])
def test_attention_layouts(swz, dim):
    """Views of one projection's rows, heads before tokens, heads that share memory: the results of dense tensors, bit for bit."""
    n, hq, hk = 190, 6, 2
    cu = cu_of([100, 90])
    rows = randn(5, n, (hq + 2 * hk) * dim)
    q, k, v = (t.view(n, -1, dim) for t in rows.split([hq * dim, hk * dim, hk * dim], 1))
    dout = randn(6, hq, n, dim).transpose(0, 1)
    want = swz.attention(q.contiguous(), k.contiguous(), v.contiguous(), cu)
    out = torch.empty((hq, n, dim), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    got = swz.attention(q, k, v, cu, out=out)
    assert got[0] is out and torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    grads = swz.attention_backward(dout.contiguous(), q.contiguous(), k.contiguous(), v.contiguous(), *want, cu)
    drows = torch.full_like(rows, float("nan"))
    parts = [t.view(n, -1, dim) for t in drows.split([hq * dim, hk * dim, hk * dim], 1)]
    swz.attention_backward(dout, q, k, v, *got, cu, None, *parts)
    assert all(torch.equal(a, b) for a, b in zip(grads, parts))
    shared = k[:, :1].expand(n, hk, dim)                       # one key head seen as two
    a, b = swz.attention(q, shared, shared, cu), swz.attention(q, shared.contiguous(), shared.contiguous(), cu)
    assert torch.equal(a[0], b[0])
    with pytest.raises(AssertionError):
        swz.attention(q, k, v, cu, out=q[:, :1].expand(n, hq, dim))


def ragged(n, seed):
    """n lengths, empty ones, single tokens and equal ones among them."""
    lens = np.random.default_rng(seed).integers(0, 90, n).tolist()
    lens[n // 2], lens[-1], lens[0] = 0, 1, lens[1]
    return lens


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("sequences", [6, 15, 16, 17, 33, 63, 64])
def test_sequences_up_to_a_lane_each(swz, sequences, dim, causal):
    """Turns of up to 16 sequences are put in order by length, those of up to 64 come from sums over lanes; the tests above have fewer, test_many_sequences more."""
    q_lens, k_lens = ragged(sequences, sequences), ragged(sequences, sequences + 100)
    k_lens[2] = k_lens[3] = max(k_lens)                         # the longest of all, twice
    nq, nk = sum(q_lens), sum(k_lens)
    q, k, v, dout = randn(nq, nq, 4, dim, scale=2.0), randn(nk, nk, 2, dim), randn(nk + 1, nk, 2, dim), randn(nq + 1, nq, 4, dim)
    for kl in (q_lens, k_lens):
        kk, vv = (k, v) if kl is k_lens else (randn(nq + 2, nq, 2, dim), randn(nq + 3, nq, 2, dim))
        cu_q, cu_k = cu_of(q_lens), cu_of(kl)
        out, lse = swz.attention(q, kk, vv, cu_q, cu_k, causal=causal)
        check_forward(q, kk, vv, out, lse, q_lens, kl, causal, dim ** -0.5)
        grads = swz.attention_backward(dout, q, kk, vv, out, lse, cu_q, cu_k, causal=causal)
        check_backward(q, kk, vv, dout, grads, q_lens, kl, causal, dim ** -0.5)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_lens,k_lens,q_heads,k_heads", [([3], [2100], 4, 1), ([33], [1300], 8, 1), ([1] * 3, [1100, 1500, 1030], 8, 2), ([40, 0, 7], [1200, 5, 3000], 12, 3)])
def test_cut_keys_of_shared_heads(swz, q_lens, k_lens, q_heads, k_heads, dim, causal):
    """Few queries over many keys, four query heads of a key head to a workgroup: the cut's parts and their join."""
    nq, nk = sum(q_lens), sum(k_lens)
    q, k, v, dout = randn(nq, nq, q_heads, dim, scale=2.0), randn(nk, nk, k_heads, dim), randn(nk + 1, nk, k_heads, dim), randn(nq + 1, nq, q_heads, dim)
    cu_q, cu_k = cu_of(q_lens), cu_of(k_lens)
    out, lse = swz.attention(q, k, v, cu_q, cu_k, causal=causal)
    check_forward(q, k, v, out, lse, q_lens, k_lens, causal, dim ** -0.5)
    check_backward(q, k, v, dout, swz.attention_backward(dout, q, k, v, out, lse, cu_q, cu_k, causal=causal), q_lens, k_lens, causal, dim ** -0.5)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_looked_at_does_not_matter(swz, dim, bad):
    """Infinities and NaN in keys and values behind the mask, in other sequences and past the end do not reach an output; those that are looked at do."""
    lens = [100, 77]
    q, k, v = randn(7, 177, 2, dim), randn(8, 177, 2, dim), randn(9, 177, 2, dim)
    cu = cu_of(lens)
    clean = swz.attention(q, k, v, cu)[0]
    k2, v2 = k.clone(), v.clone()
    k2[50:60, 0] = bad
    v2[70:100, 0] = bad
    v2[70, 1, 3] = bad
    out = swz.attention(q, k2, v2, cu)[0]
    assert torch.equal(out[:50], clean[:50]) and torch.equal(out[100:], clean[100:])
    only_v = swz.attention(q, k, v2, cu)[0]
    assert torch.isfinite(only_v[:70]).all() and (only_v[:70].float() - clean[:70].float()).abs().max() <= 2 ** -6
    assert not torch.isfinite(only_v[70:100, 0]).any() and not torch.isfinite(only_v[70:100, 1, 3]).any()
    rest = [d for d in range(dim) if d != 3]
    assert torch.isfinite(only_v[70:100, 1][:, rest]).all()
    # a buffer longer than its sequences, its rest full of what must not be seen
    long = torch.full((300, 2, dim), bad, dtype=torch.bfloat16, device="cuda")
    lk, lv = long.clone(), long.clone()
    lk[:177], lv[:177] = k, v
    # few queries and many keys, cut among workgroups
    q3, k3, v3 = randn(17, 40, 2, dim), randn(18, 1500, 2, dim), randn(19, 1500, 2, dim)
    cq, ck = cu_of([40]), cu_of([1500])
    first = swz.attention(q3, k3, v3, cq, ck)[0]
    v3[1480, 1] = bad
    got = swz.attention(q3, k3, v3, cq, ck)[0]
    assert torch.equal(got[:, 0], first[:, 0]) and torch.isfinite(got[:20, 1]).all() and not torch.isfinite(got[20:, 1]).any()
    assert (got[:20, 1].float() - first[:20, 1].float()).abs().max() <= 2 ** -6
    for causal in (True, False):
        a, b = swz.attention(q, lk, lv, cu, causal=causal), swz.attention(q, k, v, cu, causal=causal)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_lens,k_lens,q_heads,k_heads", [
    ([600], [600], 8, 1), ([333], [333], 24, 2), ([200, 0, 301, 1], [200, 0, 301, 1], 20, 1), ([500], [170], 6, 1), ([150, 250], [700, 0], 16, 1)])
def test_gradient_of_few_key_heads(swz, q_lens, k_lens, q_heads, k_heads, dim, causal):
    """A tile of keys whose queries several workgroups share: their sums are added up by another kernel."""
    nq, nk = sum(q_lens), sum(k_lens)
    q, k, v, dout = randn(nq, nq, q_heads, dim, scale=2.0), randn(nq + 1, nk, k_heads, dim), randn(nq + 2, nk, k_heads, dim), randn(nq + 3, nq, q_heads, dim)
    cu_q, cu_k = cu_of(q_lens), cu_of(k_lens)
    out, lse = swz.attention(q, k, v, cu_q, cu_k, causal=causal)
    grads = swz.attention_backward(dout, q, k, v, out, lse, cu_q, cu_k, causal=causal)
    check_backward(q, k, v, dout, grads, q_lens, k_lens, causal, dim ** -0.5)
    again = swz.attention_backward(dout, q, k, v, out, lse, cu_q, cu_k, causal=causal)
    assert all(torch.equal(a, b) for a, b in zip(again, grads))


@pytest.mark.parametrize("q_heads", [2, 16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_gradients_of_what_is_not_looked_at(swz, dim, bad, q_heads):
    """Infinities and NaN in keys, values, queries and gradients reach the gradients of what looks at them or is looked at by them, no others."""
    lens, n, group = [300, 77], 377, q_heads // 2
    q, k, v, dout = randn(7, n, q_heads, dim), randn(8, n, 2, dim), randn(9, n, 2, dim), randn(10, n, q_heads, dim)
    cu = cu_of(lens)

    def gradients(q, k, v, dout):
        return swz.attention_backward(dout, q, k, v, *swz.attention(q, k, v, cu), cu)

    clean = gradients(q, k, v, dout)

    def near(got, want):                                  # the same numbers but for the order and rounding of their sums
        return torch.isfinite(got).all() and (got.float() - want.float()).abs().max() <= 2 ** -6 * want.float().abs().max()

    for at in (40, 100, 211):
        k2, v2, q2, d2 = k.clone(), v.clone(), q.clone(), dout.clone()
        k2[at, 0] = v2[at, 0] = bad
        q2[at, 0] = bad
        d2[at, 0] = bad
        for dq, dk, dv in (gradients(q, k2, v, dout), gradients(q, k, v2, dout)):
            # queries before the key, other key heads and sequences
            assert near(dq[:at, :group], clean[0][:at, :group]) and torch.equal(dq[:, group:], clean[0][:, group:]) and torch.equal(dq[300:], clean[0][300:])
            assert not torch.isfinite(dq[at:300, :group]).any()
            assert torch.equal(dk[:, 1], clean[1][:, 1]) and torch.equal(dv[:, 1], clean[2][:, 1]) and torch.equal(dk[300:], clean[1][300:])
        for dq, dk, dv in (gradients(q2, k, v, dout), gradients(q, k, v, d2)):
            # keys behind the query, other heads and sequences
            assert near(dk[at + 1:300, 0], clean[1][at + 1:300, 0]) and near(dv[at + 1:300, 0], clean[2][at + 1:300, 0])
            assert not torch.isfinite(dk[:at + 1, 0]).any() and torch.equal(dk[:, 1], clean[1][:, 1]) and torch.equal(dv[300:], clean[2][300:])
            assert near(dq[:at, 0], clean[0][:at, 0]) and torch.equal(dq[:, 1:], clean[0][:, 1:]) and not torch.isfinite(dq[at, 0]).any()


@pytest.mark.parametrize("q_heads", [2, 8])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [1, 33, 100, 128, 190])
def test_infinities_in_the_last_token(swz, n, dim, causal, q_heads):
    """What a tile holds behind the last token must not turn an infinity of the last one, which is looked at, into NaN."""
    group = q_heads // 2
    q, k, v, dout = randn(n, n + 40, q_heads, dim), randn(n + 1, n + 40, 2, dim), randn(n + 2, n + 40, 2, dim), randn(n + 3, n + 40, q_heads, dim)
    cu = cu_of([n, 40])
    out, lse = swz.attention(q, k, v, cu, causal=causal)
    clean = swz.attention_backward(dout, q, k, v, out, lse, cu, causal=causal)
    for inf in (float("inf"), float("-inf")):
        v2, d2 = v.clone(), dout.clone()
        v2[n - 1, 0, 3] = inf
        got, lse2 = swz.attention(q, k, v2, cu, causal=causal)
        assert ((lse2 - lse).abs() <= 2e-5 * (1 + lse.abs())).all() and torch.equal(got[:, group:], out[:, group:]) and torch.equal(got[n:], out[n:])
        looks = got[n - 1 if causal else 0:n, :group]
        assert (looks[..., 3] == inf).all() and torch.isfinite(got[:n - 1 if causal else 0]).all()
        rest = [d for d in range(dim) if d != 3]
        assert (looks[..., rest].float() - out[n - 1 if causal else 0:n, :group][..., rest].float()).abs().max() <= 2 ** -6
        d2[n - 1, 0, 5] = inf
        dv = swz.attention_backward(d2, q, k, v, out, lse, cu, causal=causal)[2]
        assert (dv[:n, 0, 5] == inf).all() and torch.equal(dv[:, 1], clean[2][:, 1]) and torch.equal(dv[n:], clean[2][n:])
        rest = [d for d in range(dim) if d != 5]
        assert (dv[:n, 0][..., rest].float() - clean[2][:n, 0][..., rest].float()).abs().max() <= 2 ** -6 * clean[2].float().abs().max()


def test_distances_between_tokens(swz):
    # tiles are loaded with 32-bit offsets from their first row: longer distances are refused, not wrapped
    memory, cu = torch.zeros((1 << 28) + 64, dtype=torch.bfloat16, device="cuda"), cu_of([2])
    far, near = memory.as_strided((2, 1, 64), (1 << 28, 64, 1)), memory.as_strided((2, 1, 64), ((1 << 28) - 8, 64, 1))
    near.copy_(randn(1, 2, 1, 64))
    dense = near.contiguous()
    out, lse = swz.attention(near, near, near, cu)
    want = swz.attention(dense, dense, dense, cu)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert all(torch.equal(a, b) for a, b in zip(swz.attention_backward(near, near, near, near, out, lse, cu), swz.attention_backward(dense, dense, dense, dense, out, lse, cu)))
    for which in range(3):
        args = [dense] * 3
        args[which] = far
        with pytest.raises(swz.SwzError):
            swz.attention(*args, cu)
        with pytest.raises(swz.SwzError):
            swz.attention_backward(dense, *args, out, lse, cu)
    with pytest.raises(swz.SwzError):
        swz.attention_backward(far, dense, dense, dense, out, lse, cu)


def test_tokens_of_no_sequence_are_left_alone(swz):
    cu = torch.tensor([10, 50, 50, 90], dtype=torch.int32, device="cuda")
    q, k, v, dout = randn(1, 120, 2, 64), randn(2, 120, 1, 64), randn(3, 120, 1, 64), randn(4, 120, 2, 64)
    out, lse = torch.full_like(q, 7.0), torch.full((2, 120), 7.0, device="cuda")
    swz.attention(q, k, v, cu, out=out, lse=lse)
    inner = slice(10, 90)
    check_forward(q[inner], k[inner], v[inner], out[inner], lse[:, inner], [40, 40], [40, 40], True, 0.125)
    outs = [torch.full_like(t, 7.0) for t in (q, k, v)]
    swz.attention_backward(dout, q, k, v, out, lse, cu, None, *outs)
    check_backward(q[inner], k[inner], v[inner], dout[inner], [t[inner] for t in outs], [40, 40], [40, 40], True, 0.125)
    for t in (out, *outs, lse.t()):
        assert (t[:10] == 7).all() and (t[90:] == 7).all()


def test_lengths_that_make_no_sense_stay_inside_the_tensors(swz):
    # an end beyond the tokens, a start before them, falling starts: clamped, whatever that means for the result
    q = randn(1, 64, 1, 64)
    for cu in ([0, 1000], [-50, 30], [0, 60, 20, 64], [64, 0]):
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        out, lse = swz.attention(q, q, q, c)
        swz.attention_backward(q, q, q, q, out, lse.nan_to_num(0.0), c)
    torch.cuda.synchronize()
    out, lse = swz.attention(q, q, q, torch.tensor([0, 1000], dtype=torch.int32, device="cuda"))
    want = swz.attention(q, q, q, cu_of([64]))
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_many_sequences(swz):
    # more than the search for a tile's sequence looks at in one step, and in two
    for n in (65, 4200):
        lens = [(7 * i) % 5 for i in range(n)]
        total = sum(lens)
        q, k, v, dout = randn(n, total, 1, 64), randn(n + 1, total, 1, 64), randn(n + 2, total, 1, 64), randn(n + 3, total, 1, 64)
        cu = cu_of(lens)
        out, lse = swz.attention(q, k, v, cu)
        check_forward(q, k, v, out, lse, lens, lens, True, 0.125)
        check_backward(q, k, v, dout, swz.attention_backward(dout, q, k, v, out, lse, cu), lens, lens, True, 0.125)


def test_distances_beyond_32_bits(swz):
    n, step = 40, (1 << 32) // 32 + 8                          # the last tokens lie more than 2^32 elements behind the first
    big = torch.empty(n * step, dtype=torch.bfloat16, device="cuda")
    views = [big[i * 128:].as_strided((n, 2, 64), (step, 64, 1)) for i in range(4)]
    dense = [randn(i, n, 2, 64) for i in range(3)]
    for view, t in zip(views, dense):
        view.copy_(t)
    cu = cu_of([n])
    out, lse = swz.attention(*views[:3], cu, out=views[3])
    want = swz.attention(*dense, cu)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    grads = swz.attention_backward(views[0], *views[:3], out, lse, cu)
    assert all(torch.equal(a, b) for a, b in zip(grads, swz.attention_backward(dense[0], *dense, *want, cu)))


def test_no_tokens(swz):
    none, some = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda"), randn(0, 5, 2, 64)
    zero, five = cu_of([0]), cu_of([5])
    assert swz.attention(none, none, none, zero)[0].shape == (0, 2, 64)
    out, lse = swz.attention(some, none, none, five, zero)
    assert (out == 0).all() and torch.isneginf(lse).all()
    assert all((g == 0).all() for g in swz.attention_backward(some, some, none, none, out, lse, five, zero))
    out, lse = swz.attention(none, some, some, zero, five)
    dq, dk, dv = swz.attention_backward(none, none, some, some, out, lse, zero, five)
    assert (dk == 0).all() and (dv == 0).all() and dk.shape == some.shape


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
def test_tokens_of_no_sequence_beside_no_tokens(swz, dim, causal):
    """No keys at all, or no queries: the tokens of the sequences get 0, those of none are left alone, as ever."""
    some, none = randn(1, 8, 40, dim), torch.empty((0, 40, dim), dtype=torch.bfloat16, device="cuda")
    cu, zero = torch.tensor([2, 5], dtype=torch.int32, device="cuda"), torch.tensor([0, 0], dtype=torch.int32, device="cuda")
    inner = torch.tensor([2 <= i < 5 for i in range(8)], device="cuda")
    out, lse = torch.full_like(some, 7.0), torch.full((40, 8), 7.0, device="cuda")
    few = none[:, :1]
    swz.attention(some, few, few, cu, zero, out=out, lse=lse, causal=causal)
    assert (out[inner] == 0).all() and (out[~inner] == 7).all() and torch.isneginf(lse[:, inner]).all() and (lse[:, ~inner] == 7).all()
    dq = torch.full_like(some, 7.0)
    got = swz.attention_backward(some, some, few, few, out, lse, cu, zero, dq=dq, causal=causal)
    assert got[0] is dq and (dq[inner] == 0).all() and (dq[~inner] == 7).all() and got[1].shape == got[2].shape == few.shape
    keys = some[:, :1]
    dk, dv = torch.full((8, 1, dim), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((8, 1, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    got = swz.attention_backward(none, none, keys, keys, none, lse[:, :0].contiguous(), zero, cu, dk=dk, dv=dv, causal=causal)
    assert got[0].shape == none.shape and got[1] is dk and got[2] is dv
    for t in (dk, dv):
        assert (t[inner] == 0).all() and (t[~inner] == 7).all()
    assert [tuple(t.shape) for t in swz.attention_backward(none, none, few, few, none, lse[:, :0].contiguous(), zero, zero)] == [(0, 40, dim), (0, 1, dim), (0, 1, dim)]


@pytest.mark.parametrize("dim", [64, 128])
def test_gradient_of_no_queries_without_a_workspace(swz, dim):
    # the C call with what its own query of the size says
    import ctypes

    from paper_2508_20258_amd import attention_layer as layer

    k, v, none = randn(1, 5, 2, dim), randn(2, 5, 2, dim), torch.zeros((1, 4, dim), dtype=torch.bfloat16, device="cuda")
    dk, dv, lse = torch.full_like(k, 7.0), torch.full_like(v, 7.0), torch.zeros((4, 1), device="cuda")
    cu_q, cu_k = cu_of([0]), cu_of([5])
    h = [layer._heads(t) for t in (none, k, v, dk, dv)]
    a = layer._AttentionArgs(h[0], h[1], h[2], h[0], lse.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(), 0, 5, 1, 4, 2, dim, 1, 0.1)
    r = ctypes.byref
    assert layer.lib.swz_attention_backward_workspace(r(a)) == 0
    assert layer.lib.swz_attention_backward(r(a), r(h[0]), r(h[0]), r(h[3]), r(h[4]), None, 0, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert (dk == 0).all() and (dv == 0).all()


# ---------------------------------------------------------------- norm and rotation

def tables(rows, r, seed=0):
    a = torch.randn((rows, r // 2), generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * 3
    return a.cos().float().cuda(), a.sin().float().cuda()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,r", [(64, 64), (64, 32), (64, 16), (64, 48), (128, 128), (128, 64), (128, 16), (128, 96)])
@pytest.mark.parametrize("tokens,q_heads,k_heads", [(1, 1, 1), (2, 3, 1), (37, 8, 2), (300, 5, 5)])
def test_norm_rope_and_gradient(swz, tokens, q_heads, k_heads, dim, r, interleaved):
    seed = tokens + dim + r
    q, k = randn(seed, tokens, q_heads, dim, scale=2.0), randn(seed + 1, tokens, k_heads, dim, scale=0.1)
    wq, wk = randn(seed + 2, dim), randn(seed + 3, dim)
    dq_out, dk_out = randn(seed + 4, tokens, q_heads, dim), randn(seed + 5, tokens, k_heads, dim)
    cos, sin = tables(50, r)
    positions = torch.randint(0, 50, (tokens,), generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
    eps = 1e-3
    outs = swz.qk_norm_rope(q, k, wq, wk, cos, sin, positions, eps=eps, interleaved=interleaved)
    back = swz.qk_norm_rope_backward(dq_out, dk_out, q, k, wq, wk, cos, sin, positions, eps=eps, interleaved=interleaved)
    c, s, p = f64(cos), f64(sin), positions.cpu().numpy()
    for x, w, out, dz, dx, dw in ((q, wq, outs[0], dq_out, back[0], back[2]), (k, wk, outs[1], dk_out, back[1], back[3])):
        x, w, out, dz, dx, dw = (f64(t) for t in (x, w, out, dz, dx, dw))
        want_w, size_w = np.zeros(dim), np.zeros(dim)
        for t in range(tokens):
            want = ar.norm_rope(x[t], w, c[p[t]], s[p[t]], interleaved, eps)
            # one rounding; the two products of a turned dimension cancel, their errors do not
            size = ar.norm_rope(np.abs(x[t]), np.abs(w), np.abs(c[p[t]]), -np.abs(s[p[t]]), interleaved, eps)
            size = np.maximum(size, ar.norm_rope(np.abs(x[t]), np.abs(w), np.abs(c[p[t]]), np.abs(s[p[t]]), interleaved, eps))
            check(out[t], want, ar.ROUND * np.abs(want) + 2e-6 * size + 1e-30, f"norm of token {t}")
            wx, ww = ar.norm_rope_backward(dz[t], x[t], w, c[p[t]], s[p[t]], interleaved, eps)
            rms = np.sqrt((x[t] ** 2).mean(1, keepdims=True) + eps)
            turned = np.abs(dz[t]).max(1, keepdims=True) * 2
            most = turned * (np.abs(w).max() / rms) * (1 + np.abs(x[t]) / rms * np.sqrt(dim))
            check(dx[t], wx, ar.ROUND * np.abs(wx) + 4e-6 * most, f"gradient of token {t}")
            want_w += ww
            size_w += (turned * np.abs(x[t]) / rms).sum(0)
        check(dw, want_w, 4e-6 * size_w + 1e-30, "gradient of the weight")
    again = swz.qk_norm_rope_backward(dq_out, dk_out, q, k, wq, wk, cos, sin, positions, eps=eps, interleaved=interleaved)
    assert all(torch.equal(a, b) for a, b in zip(again, back))
    # in place, on views of one row, with the gradients in place too
    rows = torch.cat([q.flatten(1), k.flatten(1)], 1)
    vq, vk = rows[:, :q_heads * dim].view(tokens, q_heads, dim), rows[:, q_heads * dim:].view(tokens, k_heads, dim)
    gq, gk = dq_out.clone(), dk_out.clone()
    got = swz.qk_norm_rope_backward(gq, gk, vq, vk, wq, wk, cos, sin, positions, dq=gq, dk=gk, eps=eps, interleaved=interleaved)
    assert all(torch.equal(a, b) for a, b in zip(got, back)) and got[0] is gq
    swz.qk_norm_rope(vq, vk, wq, wk, cos, sin, positions, vq, vk, eps=eps, interleaved=interleaved)
    assert torch.equal(vq, outs[0]) and torch.equal(vk, outs[1])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens,q_heads,k_heads", [(1, 8, 1), (1, 32, 8), (37, 8, 2), (74, 4, 1), (129, 32, 8), (1234, 8, 3)])
def test_norm_in_place_where_the_last_workgroup_is_not_full(swz, tokens, q_heads, k_heads, dim):
    """Waves past the last head have nothing to store: one that stored what it had loaded from an output would norm it twice."""
    q, k, wq, wk = randn(tokens, tokens, q_heads, dim, scale=3.0), randn(tokens + 1, tokens, k_heads, dim), randn(2, dim), randn(3, dim)
    cos, sin = tables(50, dim)
    p = (torch.arange(tokens, device="cuda") % 50).to(torch.int32)
    want = swz.qk_norm_rope(q, k, wq, wk, cos, sin, p)
    got = swz.qk_norm_rope(q, k, wq, wk, cos, sin, p, q, k)
    assert got[0] is q and got[1] is k and torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_norm_positions_outside_the_tables(swz):
    q, w = randn(1, 6, 2, 64), randn(2, 64)
    cos, sin = tables(4, 64)
    p = torch.tensor([0, 4, 3, -1, 1 << 30, 2], dtype=torch.int32, device="cuda")
    for interleaved in (False, True):
        out, _ = swz.qk_norm_rope(q, q, w, w, cos, sin, p, interleaved=interleaved)
        assert torch.isnan(out[[1, 3, 4]]).all() and torch.isfinite(out[[0, 2, 5]]).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,r", [(64, 32), (64, 48), (128, 16), (128, 96)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("where", ["x", "gradient", "weight"])
def test_norm_of_what_is_not_finite_where_nothing_turns(swz, where, bad, dim, r, interleaved):
    """An infinity or NaN in a dimension that is not turned reaches what the formula says, not its neighbour."""
    tokens, heads, at = 5, 3, (3, 1, r + 2)
    x, dz, w = randn(dim, tokens, heads, dim), randn(dim + 1, tokens, heads, dim), randn(dim + 2, dim)
    cos, sin = tables(50, r)
    positions = torch.tensor([7, 0, 49, 23, 11], dtype=torch.int32, device="cuda")
    {"x": x[at[0], at[1]], "gradient": dz[at[0], at[1]], "weight": w}[where][at[2]] = bad
    outs = swz.qk_norm_rope(x, x, w, w, cos, sin, positions, interleaved=interleaved)
    back = swz.qk_norm_rope_backward(dz, dz, x, x, w, w, cos, sin, positions, interleaved=interleaved)
    xs, zs, ws, c, s, p = f64(x), f64(dz), f64(w), f64(cos), f64(sin), positions.cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = np.stack([ar.norm_rope(xs[t], ws, c[p[t]], s[p[t]], interleaved, 1e-6) for t in range(tokens)])
        pairs = [ar.norm_rope_backward(zs[t], xs[t], ws, c[p[t]], s[p[t]], interleaved, 1e-6) for t in range(tokens)]
        dx, dw = np.stack([g for g, _ in pairs]), sum(g for _, g in pairs)
    for side in range(2):
        for got, exact, tolerance in ((outs[side], want, ar.ROUND), (back[side], dx, ar.ROUND), (back[2 + side], dw, 1e-5)):
            got, some = f64(got), np.isfinite(exact)
            assert np.array_equal(np.isnan(got), np.isnan(exact)) and np.array_equal(got[np.isinf(exact)], exact[np.isinf(exact)])
            assert (np.abs(got[some] - exact[some]) <= 1.02 * tolerance * np.abs(exact[some]) + 1e-4).all()


def test_norm_weights_over_many_rows(swz):
    # more rows than the launch has places for: workgroups go over them in turns
    tokens, heads, dim = 40000, 8, 64
    q, dz, w = randn(1, tokens, heads, dim), randn(2, tokens, heads, dim), randn(3, dim)
    cos, sin = tables(8, 64)
    p = (torch.arange(tokens, device="cuda") % 8).to(torch.int32)
    _, _, dwq, dwk = swz.qk_norm_rope_backward(dz, dz[:, :1], q, q[:, :1], w, w, cos, sin, p)
    x, g, c, s = q.double(), dz.double(), cos.double()[p.long()][:, None], sin.double()[p.long()][:, None]
    g = torch.cat([g[..., :32] * c + g[..., 32:] * s, g[..., 32:] * c - g[..., :32] * s], -1)
    terms = g * x / ((x * x).mean(-1, keepdim=True) + 1e-6).sqrt()
    for got, want in ((dwq, terms), (dwk, terms[:, :1])):
        assert ((got.double() - want.sum((0, 1))).abs() <= 4e-6 * want.abs().sum((0, 1))).all()


# ---------------------------------------------------------------- the cache

def table_of(lens, page, seed=0, width=None):
    need = [-(-n // page) for n in lens]
    order = np.random.default_rng(seed).permutation(sum(need) + 3)
    table = np.full((len(lens), width or max(max(need), 1)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return torch.from_numpy(table).cuda(), sum(need) + 3


def poison(cache):
    """What uninitialised memory may hold."""
    for t in cache:
        t.view(torch.int16).fill_(-1)


def numbers_of(cache, table, lens, page):
    """(step, low, n) arrays (tokens, heads, dim) of K and V for each sequence, read from the words by their definition."""
    out = []
    k_words, v_words = (t.cpu().numpy().view(np.uint32) for t in (cache.k_words, cache.v_words))
    scales = [f64(t) for t in (cache.k_scales, cache.v_scales)]
    heads, dim = k_words.shape[1], k_words.shape[3] * 8
    shift = [4 * (e // 2 + 4 * (e % 2)) for e in range(8)]
    for b, n in enumerate(lens):
        res = [np.zeros((n, heads, dim)) for _ in range(6)]
        for t in range(n):
            p, i = int(table[b, t // page]), t % page
            for d in range(dim):
                word = k_words[p, :, i, dim // 32 * (d % 32 // 8) + d // 32]
                res[2][t, :, d] = word >> shift[d % 8] & 15
            res[5][t] = v_words[p, :, i // 8, :] >> shift[i % 8] & 15
            for which in range(2):
                for part in range(2):
                    res[3 * which + part][t] = np.repeat(scales[which][p, :, i, :, part], 64, axis=-1)
        out.append(res)
    return out


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [32, 64, 256])
@pytest.mark.parametrize("lens,before", [([1], [0]), ([9, 0, 70], [3, 5, 0]), ([64, 33, 8], [7, 31, 8]), ([300], [0])])
def test_cache_append_and_read(swz, lens, before, page, dim):
    heads, n = 3, sum(lens)
    k, v = randn(n + page, n, heads, dim) + 1.5, randn(n + 1, n, heads, dim, scale=3.0)
    k[0, 0] = 2.5                                               # a group of one value
    v[0, 1, 5] = float("nan")
    v[0, 2, 63] = float("-inf")
    if n > 1:
        k[1, 0, :64:2], k[1, 0, 1:64:2] = 3e38, -3e38            # a range that is no number
    ends = [a + m for a, m in zip(before, lens)]
    table, pages = table_of(ends, page)
    cache = swz.kv_cache4(pages, heads, dim, page)
    poison(cache)
    b = torch.tensor(before, dtype=torch.int32, device="cuda")
    old_k, old_v = randn(77, sum(before), heads, dim), randn(78, sum(before), heads, dim)
    if sum(before):
        swz.cache4_append(cache, old_k, old_v, cu_of(before), torch.zeros_like(b), table)
    swz.cache4_append(cache, k, v, cu_of(lens), b, table)
    got = swz.cache4_read(cache, cu_of(ends), torch.zeros_like(b), table, sum(ends))
    held = numbers_of(cache, table, ends, page)
    at, first, new = 0, 0, 0
    for s, (m, a) in enumerate(zip(lens, before)):
        for which, (fresh, old) in enumerate(((k, old_k), (v, old_v))):
            x = torch.cat([old[first:first + a], fresh[new:new + m]]).float().cpu().numpy()
            step, low, num = held[s][3 * which:3 * which + 3]
            value = f64(got[which][at:at + a + m])
            for t in range(a + m):
                for h in range(heads):
                    for g in range(dim // 64):
                        want = ar.quantise(x[t, h, 64 * g:64 * g + 64])
                        here = (t, h, slice(64 * g, 64 * g + 64))
                        assert np.array_equal(step[here], np.full(64, want[0], dtype=np.float64), equal_nan=True)
                        assert np.array_equal(low[here], np.full(64, want[1], dtype=np.float64), equal_nan=True)
                        if not np.isnan(want[0]):
                            assert np.array_equal(num[here], want[2])
                        assert np.array_equal(value[here], ar.to_bf16(want[1] + want[0] * want[2]).astype(np.float64), equal_nan=True)
        at, first, new = at + a + m, first + a, new + m
    # a part of it, from the middle of a word
    part = [max(0, e - 5) for e in ends]
    some = [min(5, e) for e in ends]
    mid = swz.cache4_read(cache, cu_of(some), torch.tensor(part, dtype=torch.int32, device="cuda"), table, sum(some))
    at = o = 0
    for e, p, m in zip(ends, part, some):
        for which in range(2):
            assert torch.equal(mid[which][o:o + m].nan_to_num(9.0), got[which][at + p:at + p + m].nan_to_num(9.0))
        at, o = at + e, o + m


def test_cache_layouts_and_pages_that_are_not_there(swz):
    heads, dim, page = 2, 128, 32
    lens = [40, 50]
    rows = randn(1, 90, 2 * heads * dim)
    k, v = rows[:, :heads * dim].view(90, heads, dim), rows[:, heads * dim:].view(90, heads, dim)
    zero, cu = torch.zeros(2, dtype=torch.int32, device="cuda"), cu_of(lens)
    table, pages = table_of(lens, page)
    a, b = swz.kv_cache4(pages, heads, dim, page), swz.kv_cache4(pages, heads, dim, page)
    swz.cache4_append(a, k, v, cu, zero, table)
    swz.cache4_append(b, k.contiguous(), v.contiguous(), cu, zero, table)
    assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(a, b))
    back = swz.cache4_read(a, cu, zero, table, 90)
    out = torch.empty_like(rows)
    ok, ov = out[:, :heads * dim].view(90, heads, dim), out[:, heads * dim:].view(90, heads, dim)
    swz.cache4_read(a, cu, zero, table, 90, ok, ov)
    assert torch.equal(ok, back[0]) and torch.equal(ov, back[1])
    # entries that name no page, positions past the table, starts that make no sense: nothing is written, NaN is read
    wrong = table.clone()
    wrong[0, 1], wrong[1, 0] = pages, -1
    before = [x.clone() for x in a]
    swz.cache4_append(a, k + 1, v + 1, cu, zero, wrong)
    held = swz.cache4_read(a, cu, zero, wrong, 90)
    assert torch.isnan(held[0][32:72]).all() and torch.isnan(held[1][32:72]).all() and torch.isfinite(held[0][:32]).all() and torch.isfinite(held[1][72:]).all()
    changed = {int(table[0, 0]), int(table[1, 1])}
    for x, y in zip(a, before):
        for p in range(pages):
            assert (p in changed) or torch.equal(x[p].view(torch.int16), y[p].view(torch.int16))
    for start in (64, 1 << 30, -3, (1 << 31) - 1):
        s = torch.tensor([start, start], dtype=torch.int32, device="cuda")
        before = [x.clone() for x in a]
        swz.cache4_append(a, k, v, cu, s, table)
        assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(a, before))
    s = torch.full((2,), 64, dtype=torch.int32, device="cuda")
    assert torch.isnan(swz.cache4_read(a, cu, s, table, 90)[0]).all()


def decode_case(swz, lens, q_heads, k_heads, dim, page, seed=0):
    table, pages = table_of(lens, page, seed)
    cache = swz.kv_cache4(pages, k_heads, dim, page)
    poison(cache)
    n = sum(lens)
    k, v = randn(seed, n, k_heads, dim) + randn(seed + 1, 1, k_heads, dim), randn(seed + 2, n, k_heads, dim)
    zero = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    swz.cache4_append(cache, k, v, cu_of(lens), zero, table)
    return cache, table, randn(seed + 3, len(lens), q_heads, dim, scale=1.5)


def check_decode(got, q, held, lens, k_heads, scale):
    got, q = f64(got), f64(q)
    group = q.shape[1] // k_heads
    for b, n in enumerate(lens):
        ks, kl, kn, vs, vl, vn = held[b]
        for h in range(q.shape[1]):
            kh = h // group
            want, bound = ar.decode(q[b, h], (kl + ks * kn)[:, kh], (vl + vs * vn)[:, kh], vs[:, kh], vn[:, kh], scale)
            check(got[b, h], want, bound, f"sequence {b}, head {h}")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,q_heads,k_heads,page", [([1], 1, 1, 32), ([0, 1, 2, 31], 4, 2, 32), ([32, 33, 65, 127], 6, 2, 64), ([300, 0, 511], 8, 1, 64), ([700], 17, 1, 256),
                                                       ([129, 1000], 40, 1, 32), ([2500], 3, 3, 64)])
def test_cache_attention(swz, lens, q_heads, k_heads, page, dim):
    cache, table, q = decode_case(swz, lens, q_heads, k_heads, dim, page, seed=sum(lens) + dim)
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    held = numbers_of(cache, table, lens, page)
    for longest in (0, max(lens), 1):                          # unknown, known, and said too short
        got = swz.cache4_attention(q, cache, lengths, table, longest)
        check_decode(got, q, held, lens, k_heads, dim ** -0.5)
        assert torch.equal(got, swz.cache4_attention(q, cache, lengths, table, longest))
    wide = torch.cat([q, q], 1)[:, :q_heads]                   # not dense
    out = torch.empty((q_heads, len(lens), dim), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert torch.equal(swz.cache4_attention(wide, cache, lengths, table, max(lens), out=out), swz.cache4_attention(q, cache, lengths, table, max(lens)))
    # lengths below 0 and beyond the table
    odd = swz.cache4_attention(q, cache, torch.full_like(lengths, -5), table)
    assert (odd == 0).all()
    if len(lens) == 1 and table.shape[1] * page == lens[0]:
        assert torch.equal(swz.cache4_attention(q, cache, lengths + 1000, table), swz.cache4_attention(q, cache, lengths, table))


def test_cache_attention_split_over_a_long_table(swz):
    # a table far wider than the sequences: parts that have no tokens
    lens, dim, page = [5, 900, 0], 128, 64
    cache, table, q = decode_case(swz, lens, 4, 2, dim, page)
    wide = torch.full((3, 3000), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    held = numbers_of(cache, table, lens, page)
    for longest in (0, 900, 100000):
        check_decode(swz.cache4_attention(q, cache, lengths, wide, longest), q, held, lens, 2, dim ** -0.5)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_heads,k_heads", [(1, 1), (8, 2), (15, 3), (16, 2), (40, 2)])
@pytest.mark.parametrize("lens", [[1], [64], [65, 0, 127], [700, 3], [1025, 2049, 0, 0, 130], [5] * 70])
def test_cache_attention_by_workgroups_and_by_waves(swz, lens, q_heads, k_heads, dim):
    """Short sequences have a workgroup each, where the longest length says so; else waves share the steps of all sequences.  Both on the same cache."""
    page = 64
    cache, table, q = decode_case(swz, lens, q_heads, k_heads, dim, page, seed=sum(lens) + q_heads)
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    held = numbers_of(cache, table, lens, page)
    for longest in (64, 1 << 20):
        wide = torch.full((len(lens), max(table.shape[1], 40)), -1, dtype=torch.int32, device="cuda")
        wide[:, :table.shape[1]] = table
        got = swz.cache4_attention(q, cache, lengths, wide, longest)
        check_decode(got, q, held, lens, k_heads, dim ** -0.5)


def test_cache_attention_sees_nothing_else(swz):
    lens, dim, page = [70, 33], 64, 32
    cache, table, q = decode_case(swz, lens, 2, 1, dim, page)
    lengths = torch.tensor([69, 33], dtype=torch.int32, device="cuda")
    want = swz.cache4_attention(q, cache, lengths, table)
    last = int(table[0, 2])
    cache.v_scales[last, :, 5:] = float("nan")                 # position 69 and what lies behind it
    cache.k_scales[last, :, 5:] = float("inf")
    assert torch.equal(swz.cache4_attention(q, cache, lengths, table), want)
    lengths[0] = 70
    got = swz.cache4_attention(q, cache, lengths, table)
    assert torch.isnan(got[0]).all() and torch.equal(got[1], want[1])
    lengths[0] = 69
    wrong = table.clone()
    wrong[0, 1] = 1 << 30
    got = swz.cache4_attention(q, cache, lengths, wrong)
    assert torch.isnan(got[0]).all() and torch.equal(got[1], want[1])


def test_cache_words_beyond_32_bits(swz):
    # the last pages lie more than 2^32 bytes behind the first
    heads, dim, page = 8, 128, 64
    pages = (1 << 32) // (heads * page * dim // 2) + 40
    cache = swz.kv_cache4(pages, heads, dim, page)
    lens = [130, 64]
    table = torch.tensor([[pages - 1, pages - 7, 3], [pages - 2, -1, -1]], dtype=torch.int32, device="cuda")
    near = torch.tensor([[0, 1, 2], [3, -1, -1]], dtype=torch.int32, device="cuda")
    small = swz.kv_cache4(4, heads, dim, page)
    k, v, q = randn(1, 194, heads, dim), randn(2, 194, heads, dim), randn(3, 2, 2 * heads, dim)
    zero, lengths = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
    for c, t in ((cache, table), (small, near)):
        swz.cache4_append(c, k, v, cu_of(lens), zero, t)
    assert all(torch.equal(a, b) for a, b in zip(swz.cache4_read(cache, cu_of(lens), zero, table, 194), swz.cache4_read(small, cu_of(lens), zero, near, 194)))
    assert torch.equal(swz.cache4_attention(q, cache, lengths, table), swz.cache4_attention(q, small, lengths, near))


@pytest.mark.parametrize("dim", [64, 128])
def test_cache_attention_of_the_longest_table(swz, dim):
    """All positions that a table may have, in one page that it names over and over: the weights of the page's tokens are those of the page alone, and so is the result."""
    page = 1024
    cache, _, q = decode_case(swz, [page], 4, 1, dim, page)
    cache = swz.Cache4(*(t[:1].contiguous() for t in cache))
    k, v = randn(1, page, 1, dim), randn(2, page, 1, dim)
    one = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    swz.cache4_append(cache, k, v, cu_of([page]), one[0], one)
    table = torch.zeros((1, ((1 << 31) - 4096) // page), dtype=torch.int32, device="cuda")
    held = numbers_of(cache, one, [page], page)
    for n in (1, 2, table.shape[1] - 1, table.shape[1]):
        lengths = torch.tensor([n * page], dtype=torch.int32, device="cuda")
        check_decode(swz.cache4_attention(q, cache, lengths, table), q, held, [page], 1, dim ** -0.5)
    got = swz.cache4_attention(q, cache, torch.full_like(lengths, (1 << 31) - 1), table)       # cut to the table
    assert torch.equal(got, swz.cache4_attention(q, cache, lengths, table))


@pytest.mark.parametrize("q_heads,k_heads,dim,times", [(1, 1, 128, 256), (32, 8, 128, 256), (16, 16, 64, 256), (64, 64, 128, 64)])
def test_cache_attention_of_long_contexts(swz, q_heads, k_heads, dim, times):
    """1024 tokens, named up to 262144 / 1024 times by a table: the exact result does not change, and no error may grow with the number of steps that a wave adds up.

    Root mean squares.  A rounded weight is off by 2^-9 / sqrt(3) of itself on average, and multiplies a number of 4.6 steps (0..15, less 8) of 0.31 deviations each:
    0.0016 of the values, which the sum over tokens keeps in proportion to their own sum; rounding the result adds 0.0011: 0.0019.  Twice that."""
    page, n = 64, 1024
    table, pages = table_of([n], page, 1)
    cache = swz.kv_cache4(pages, k_heads, dim, page)
    k, v = randn(1, n, k_heads, dim), randn(2, n, k_heads, dim)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    swz.cache4_append(cache, k, v, cu_of([n]), zero, table)
    (ks, kl, kn, vs, vl, vn), = numbers_of(cache, table, [n], page)
    keys, values = (kl + ks * kn).transpose(1, 0, 2), (vl + vs * vn).transpose(1, 0, 2)
    for scale in (0.0, 0.3, 1.5):                              # of the queries: flat weights, and peaked ones
        q = randn(3, 1, q_heads, dim, scale=scale)
        s = f64(q)[0].reshape(k_heads, -1, dim) @ keys.transpose(0, 2, 1) * dim ** -0.5
        p = np.exp(s - s.max(-1, keepdims=True))
        want = ((p / p.sum(-1, keepdims=True)) @ values).reshape(q_heads, dim)
        for m in (1, times // 16, times):
            got = f64(swz.cache4_attention(q, cache, torch.full_like(zero, m * n), table.repeat(1, m)))[0]
            assert np.sqrt(((got - want) ** 2).mean()) <= 0.0038 * np.sqrt((want ** 2).mean()), (scale, m)


# ---------------------------------------------------------------- streams and graphs

def layer_pass(swz, t, stream=None):
    q, k = swz.qk_norm_rope(t["q"], t["k"], t["w"], t["w"], t["cos"], t["sin"], t["p"], stream=stream)
    out, lse = swz.attention(q, k, t["v"], t["cu"], stream=stream)
    grads = swz.attention_backward(t["dout"], q, k, t["v"], out, lse, t["cu"], stream=stream)
    back = swz.qk_norm_rope_backward(grads[0], grads[1], t["q"], t["k"], t["w"], t["w"], t["cos"], t["sin"], t["p"], stream=stream)
    swz.cache4_append(t["cache"], k, t["v"], t["cu"], t["zero"], t["table"], stream=stream)
    held = swz.cache4_read(t["cache"], t["cu"], t["zero"], t["table"], 160, stream=stream)
    one = swz.cache4_attention(q[:2], t["cache"], t["lengths"], t["table"], stream=stream)
    return [out, lse, *grads, *back, *held, one]


def layer_inputs(swz, seed):
    table, pages = table_of([100, 60], 64)
    cos, sin = tables(100, 128)
    return dict(q=randn(seed, 160, 4, 128), k=randn(seed + 1, 160, 2, 128), v=randn(seed + 2, 160, 2, 128), w=randn(seed + 3, 128), dout=randn(seed + 4, 160, 4, 128), cos=cos, sin=sin,
                p=torch.cat([torch.arange(100), torch.arange(60)]).to(torch.int32).cuda(), cu=cu_of([100, 60]), zero=torch.zeros(2, dtype=torch.int32, device="cuda"), table=table,
                cache=swz.kv_cache4(pages, 2, 128), lengths=torch.tensor([100, 60], dtype=torch.int32, device="cuda"))


def test_another_stream(swz):
    t = layer_inputs(swz, 1)
    want = layer_pass(swz, t)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = layer_pass(swz, t, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):
        got = layer_pass(swz, t)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_stream_that_is_a_handle_alone(swz):
    class Handle:
        def __init__(self, stream):
            self.cuda_stream = stream.cuda_stream

    t = layer_inputs(swz, 2)
    want = layer_pass(swz, t)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, torch.cuda.default_stream()):
        got = layer_pass(swz, t, stream=Handle(stream))
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_memory_still_in_use_on_the_current_stream(swz):
    """Blocks that were freed on the current stream while work on it waits, of the sizes that a pass makes: the pass on another stream gets none of them."""
    t = layer_inputs(swz, 3)
    want = layer_pass(swz, t)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    for _ in range(3):
        junk = [torch.empty_like(x) for x in want] + [torch.empty(1 << n, dtype=torch.uint8, device="cuda") for n in range(9, 21)]
        for x in junk:
            x.fill_(77)
        del junk, x
    got = layer_pass(swz, t, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_in_a_graph(swz):
    t = layer_inputs(swz, 5)
    layer_pass(swz, t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer_pass(swz, t)
    for seed in (11, 12, 13):
        fresh = layer_inputs(swz, seed)
        for name in ("q", "k", "v", "w", "dout"):
            t[name].copy_(fresh[name])
        graph.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in got]
        want = layer_pass(swz, t)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, want))
