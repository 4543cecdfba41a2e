"""The operators of an attention layer as they are measured on one MI355X: the norm and rotation of queries and keys, attention over packed
prompts, forward and backward, and attention over a cache held in 4 bits.

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes what a program has in hand before the call, `run()` is
one pass, `work()` its minimal traffic and arithmetic, `exact()` the same result in 64 bits.  With `own` false `run()` computes the plain form
from elementary torch operations in 32 bits, with `own` true it calls the package.

Sequences are packed: tokens of all sequences one after the other, `cu` their first tokens and the total.  The cache holds 64 values of a head
as 4-bit numbers n with a bfloat16 step and low each, value = low + step * n; the layout of its words is in `quantise` and `cache_values`.
"""
import math
import random

import torch

own = False

GROUP = 64                       # values of a head that share a step and a low
PAGE = 64                        # tokens of a page
EPS = 1e-6

# what a drawn case costs at most, no more than the largest listed one of its kind
MAX_NORM = 32768 * 40 * 128      # elements of queries and keys
MAX_NORM_BACK = 12345 * 40 * 128
MAX_PROMPT = 16 * 128 * 32768 * 32769 // 2   # heads * head size * pairs of a query and a key
MAX_TRAIN = 32 * 128 * 8192 * 8193 // 2
MAX_STORE = 32768 * 8 * 128
MAX_DECODE = 64 * 8192 * 8 * 128             # values of K in the cache


def listed():
    return [
        # one step of a batch of 16 sequences: the launch is most of it
        dict(name="norm_tokens", op="norm", T=16, Hq=32, Hk=8, D=128, R=128, interleaved=False),
        # the tokens of long prompts, queries and keys where the projection left them (rows of queries, keys and values)
        dict(name="norm_prompt", op="norm", T=32768, Hq=32, Hk=8, D=128, R=128, interleaved=False),
        # the gradient for a batch of packed sequences; and with small heads of which half is rotated, in pairs of neighbours
        dict(name="norm_back", op="norm_back", T=12345, Hq=32, Hk=8, D=128, R=128, interleaved=False),
        dict(name="norm_back_64", op="norm_back", T=4096, Hq=16, Hk=16, D=64, R=32, interleaved=True),
        # prompts: a batch of short ones of all lengths, one of them empty; one long one; the next pieces of prompts whose first parts are
        # there already (fewer queries than keys), one with fewer keys than queries, whose first rows have nothing to look at
        dict(name="prompt_short", op="prompt", Hq=32, Hk=8, D=128, causal=True, q_lens=_text(_ragged(5, 48, 1, 512) + [0, 1, 512]), k_lens=""),
        dict(name="prompt_long", op="prompt", Hq=16, Hk=4, D=128, causal=True, q_lens="32768", k_lens=""),
        dict(name="prompt_pieces", op="prompt", Hq=32, Hk=8, D=64, causal=True, q_lens="512,2048,1000,300,1", k_lens="8192,2048,10000,200,4096"),
        # training steps, forward and backward: packed sequences of different lengths, shared key heads; and a full batch of equal ones with as
        # many key heads as query heads
        dict(name="train_packed", op="train", Hq=32, Hk=8, D=128, causal=True, q_lens="4096,2500,1023,7,600,1", k_lens=""),
        dict(name="train_64", op="train", Hq=16, Hk=16, D=64, causal=True, q_lens="2048,2048,2048,2048", k_lens=""),
        # a prompt's keys and values into the cache and back out of it, for the next piece of the prompt
        dict(name="store", op="store", Hk=8, D=128, q_lens="10000,4096,333,1,2048", before="0,100,7,63,4096"),
        # single tokens against the cache: a few short sequences, where latency counts; a full batch of all lengths
        dict(name="decode_small", op="decode", Hq=32, Hk=8, D=128, lens="1000,512,1,0"),
        dict(name="decode_batch", op="decode", Hq=32, Hk=8, D=128, lens=_text(_ragged(9, 63, 512, 8192) + [8192])),
    ]


def _ragged(seed, n, lo, hi):
    rng = random.Random(seed)
    return [_log_int(rng, lo, hi) for _ in range(n)]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _text(lens):
    return ",".join(str(n) for n in lens)


def _ints(text):
    return [int(n) for n in text.split(",")]


def _heads(rng):
    Hk = rng.choice([1, 2, 4, 8, 16])
    return Hk * rng.choice([g for g in (1, 2, 3, 4, 6, 8) if g * Hk <= 64]), Hk


def draw(rng):
    op = rng.choice(["norm", "norm_back", "prompt", "prompt", "train", "train", "store", "decode", "decode"])
    D = rng.choice([64, 128, 128])
    while True:
        Hq, Hk = _heads(rng)
        if op in ("norm", "norm_back"):
            T = _log_int(rng, 1, 65536)
            if T * (Hq + Hk) * D <= (MAX_NORM if op == "norm" else MAX_NORM_BACK):
                return dict(op=op, T=T, Hq=Hq, Hk=Hk, D=D, R=rng.choice([D, D, D // 2, 16]), interleaved=rng.random() < 0.3)
        if op in ("prompt", "train"):
            n = _log_int(rng, 1, 64)
            longest = _log_int(rng, 16, 32768 if op == "prompt" else 8192)
            q_lens = [_log_int(rng, 1, longest) for _ in range(n)]
            k_lens = [k if rng.random() < 0.1 else q + k for q, k in zip(q_lens, (_log_int(rng, 1, longest) for _ in q_lens))] if op == "prompt" and rng.random() < 0.3 else None
            case = dict(op=op, Hq=Hq, Hk=Hk, D=D, causal=rng.random() < 0.8, q_lens=_text(q_lens), k_lens=_text(k_lens) if k_lens else "")
            if Hq * D * sum(_pairs(case)) <= (MAX_PROMPT if op == "prompt" else MAX_TRAIN) and sum(k_lens or q_lens) <= 65536:
                return case
        if op == "store":
            n = _log_int(rng, 1, 64)
            q_lens = [_log_int(rng, 1, 16384) for _ in range(n)]
            if sum(q_lens) * Hk * D <= MAX_STORE:
                return dict(op=op, Hk=Hk, D=D, q_lens=_text(q_lens), before=_text([rng.choice([0, _log_int(rng, 1, 4096)]) for _ in q_lens]))
        if op == "decode":
            n = _log_int(rng, 1, 128)
            longest = _log_int(rng, 16, 262144)
            lens = [_log_int(rng, 1, longest) for _ in range(n)]
            if sum(lens) * Hk * D <= MAX_DECODE:
                return dict(op=op, Hq=Hq, Hk=Hk, D=D, lens=_text(lens))


def _lens(case):
    q = _ints(case["q_lens"])
    return q, _ints(case["k_lens"]) if case.get("k_lens") else q


def _pairs(case):
    """For each sequence how many pairs of a query and a key that it may look at.  Causal: the last query looks at all keys, each one before at one fewer."""
    out = []
    for q, k in zip(*_lens(case)):
        if not case["causal"]:
            out.append(q * k)
        else:
            rows = min(q, k)                       # queries that look at anything
            out.append(rows * k - rows * (rows - 1) // 2)
    return out


def work(case):
    op, D, Hk = case["op"], case["D"], case["Hk"]
    if op == "norm":
        T, H = case["T"], case["Hq"] + Hk
        return {"bytes": 4 * T * H * D + 4 * T * case["R"] + 4 * T + 4 * D, "flops": 8 * T * H * D}
    if op == "norm_back":
        T, H = case["T"], case["Hq"] + Hk
        return {"bytes": 6 * T * H * D + 4 * T * case["R"] + 4 * T + 12 * D, "flops": 16 * T * H * D}
    if op in ("prompt", "train"):
        q_lens, k_lens = _lens(case)
        q, k = sum(q_lens) * case["Hq"] * D, sum(k_lens) * Hk * D
        p = sum(_pairs(case)) * case["Hq"] * D
        if op == "prompt":
            return {"bytes": 2 * (2 * q + 2 * k), "flops": 4 * p}
        return {"bytes": 2 * (4 * q + 4 * k), "flops": 14 * p}           # 2 products forward, 5 backward
    cached = D // 2 + 4 * (D // GROUP)                                   # bytes of a head's keys, or values, of one token
    if op == "store":
        n = sum(_ints(case["q_lens"])) * Hk
        return {"bytes": n * (2 * 2 * 2 * D + 2 * 2 * cached), "flops": 2 * n * 6 * D}
    n = sum(_ints(case["lens"]))
    B = len(_ints(case["lens"]))
    return {"bytes": n * Hk * 2 * cached + B * case["Hq"] * D * 4, "flops": 4 * n * case["Hq"] * D}


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, scale=1.0):
    """bfloat16 normal values, made in strips: the 32-bit values of a large tensor need not exist at once."""
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, device="cuda", generator=g) * scale
    return out


def _cu(lens):
    return torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)


def quantise(x):
    """x (..., 64), 32-bit: step, low (...) and n (..., 64).  A group whose range is no finite number has step and low NaN."""
    low, high = x.amin(-1), x.amax(-1)
    step = ((high - low) / 15).to(torch.bfloat16)
    bad = ~torch.isfinite(high - low)
    step[bad] = math.nan
    low = low.to(torch.bfloat16)
    low[bad] = math.nan
    s = step.float()[..., None]
    n = torch.where(s > 0, torch.round((x - low.float()[..., None]) / s), torch.zeros_like(x)).clamp(0, 15).to(torch.int32)
    return step, low, n


def _pack(n):
    """(..., 8) numbers of 0..15 to one 32-bit word: number 2 i + h in bits 4 (i + 4 h) and up."""
    word = torch.zeros(n.shape[:-1], dtype=torch.int32, device=n.device)
    for i in range(4):
        for h in range(2):
            word |= n[..., 2 * i + h] << (4 * (i + 4 * h))
    return word


def _unpack(word):
    return torch.stack([(word >> (4 * (i + 4 * h))) & 15 for i in range(4) for h in range(2)], -1)


def _k_words(n):
    """n (..., D) to (..., D / 8) words: word (D / 32) g + s of a key holds its numbers 32 s + 8 g and up."""
    D = n.shape[-1]
    return _pack(n.view(*n.shape[:-1], D // 32, 4, 8)).transpose(-1, -2).reshape(*n.shape[:-1], D // 8)


def _k_numbers(words):
    D = words.shape[-1] * 8
    return _unpack(words.view(*words.shape[:-1], 4, D // 32).transpose(-1, -2)).reshape(*words.shape[:-1], D)


def _v_words(n):
    """n (..., tokens, D) to (..., tokens / 8, D) words of 8 tokens of one dimension each."""
    return _pack(n.view(*n.shape[:-2], n.shape[-2] // 8, 8, n.shape[-1]).transpose(-1, -2))


def _v_numbers(words):
    return _unpack(words).transpose(-1, -2).reshape(*words.shape[:-2], words.shape[-2] * 8, words.shape[-1])


def _empty_cache(pages, Hk, D):
    z = dict(dtype=torch.int32, device="cuda")
    return dict(k_words=torch.zeros((pages, Hk, PAGE, D // 8), **z), v_words=torch.zeros((pages, Hk, PAGE // 8, D), **z),
                k_scales=torch.zeros((pages, Hk, PAGE, D // GROUP, 2), dtype=torch.bfloat16, device="cuda"),
                v_scales=torch.zeros((pages, Hk, PAGE, D // GROUP, 2), dtype=torch.bfloat16, device="cuda"))


def _table(g, lens):
    """Pages of each sequence, in no order; entries past a sequence's end are -1."""
    need = [-(-n // PAGE) for n in lens]
    order = torch.randperm(max(1, sum(need)), device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(lens), max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    first = 0
    for b, n in enumerate(need):
        table[b, :n] = order[first:first + n]
        first += n
    return table, max(1, sum(need))


def _inputs(case, seed):
    g = _generator(seed)
    op, D, Hk = case["op"], case["D"], case["Hk"]
    s = dict(case=case)
    if op in ("norm", "norm_back"):
        T, Hq, R = case["T"], case["Hq"], case["R"]
        qkv = _normal(g, (T, (Hq + 2 * Hk) * D), 1.5)                    # the rows that a projection writes
        s["q"] = qkv[:, :Hq * D].view(T, Hq, D)
        s["k"] = qkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
        s["q_weight"], s["k_weight"] = 1 + 0.2 * _normal(g, (D,)), 1 + 0.2 * _normal(g, (D,))
        angle = torch.arange(8192, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(0, R, 2, device="cuda").double() / R)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["positions"] = torch.randint(0, 8192, (T,), device="cuda", generator=g, dtype=torch.int32)
        if op == "norm_back":
            s["dq"], s["dk"] = _normal(g, (T, Hq, D)), _normal(g, (T, Hk, D))
    elif op in ("prompt", "train"):
        q_lens, k_lens = _lens(case)
        Hq = case["Hq"]
        s["q"] = _normal(g, (sum(q_lens), Hq, D), 1.5)                   # scores of a spread of 1.5
        s["k"], s["v"] = _normal(g, (sum(k_lens), Hk, D)), _normal(g, (sum(k_lens), Hk, D))
        s["cu_q"], s["cu_k"] = _cu(q_lens), _cu(k_lens)
        if op == "train":
            s["dout"] = _normal(g, (sum(q_lens), Hq, D))
    elif op == "store":
        lens, before = _ints(case["q_lens"]), _ints(case["before"])
        s["k"], s["v"] = _normal(g, (sum(lens), Hk, D)) + 0.5 * _normal(g, (Hk, D)), _normal(g, (sum(lens), Hk, D))
        s["cu_q"] = _cu(lens)
        s["before"] = torch.tensor(before, dtype=torch.int32, device="cuda")
        s["table"], pages = _table(g, [a + n for a, n in zip(before, lens)])
        s["cache"] = _empty_cache(pages, Hk, D)
    else:
        lens = _ints(case["lens"])
        s["table"], pages = _table(g, lens)
        s["cache"] = c = _empty_cache(pages, Hk, D)
        offset = 0.5 * _normal(g, (1, Hk, 1, D)).float()
        strip = max(1, (1 << 25) // (Hk * PAGE * D))
        for i in range(0, pages, strip):
            n = min(strip, pages - i)
            for name in ("k", "v"):
                x = torch.randn((n, Hk, PAGE, D), device="cuda", generator=g)
                x = (x + offset if name == "k" else x).to(torch.bfloat16).float()
                step, low, codes = quantise(x.view(n, Hk, PAGE, D // GROUP, GROUP))
                c[name + "_words"][i:i + n] = (_k_words if name == "k" else _v_words)(codes.view(n, Hk, PAGE, D))
                c[name + "_scales"][i:i + n, ..., 0] = step
                c[name + "_scales"][i:i + n, ..., 1] = low
        s["q"] = _normal(g, (len(lens), case["Hq"], D), 1.5)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["max_len"] = max(lens)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and "cache" in s:
        import paper_2508_20258_amd as swz
        s["cache"] = swz.Cache4(**s["cache"])
    return s


# ---------------------------------------------------------------- the plain forms

def _norm(x, weight):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()


def _turn(y, cos, sin, interleaved):
    """y (T, H, D): the pairs of its first R dimensions turned by the angles of the token; R / 2 = the angles of cos and sin (T, R / 2)."""
    h = cos.shape[-1]
    a, b = (y[..., 0:2 * h:2], y[..., 1:2 * h:2]) if interleaved else (y[..., :h], y[..., h:2 * h])
    c, s = cos[:, None], sin[:, None]
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, y[..., 2 * h:]), -1)


def _plain_norm(s):
    c, n = s["cos"][s["positions"].long()], s["sin"][s["positions"].long()]
    return tuple(_turn(_norm(s[x], s[x + "_weight"]), c, n, s["case"]["interleaved"]).to(torch.bfloat16) for x in ("q", "k"))


def _plain_norm_back(s):
    c, n = s["cos"][s["positions"].long()], s["sin"][s["positions"].long()]
    outs, weights = [], []
    for name in ("q", "k"):
        x = s[name].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        unit = x * r
        dy = _turn(s["d" + name].float(), c, -n, s["case"]["interleaved"])          # turned back
        weights.append((dy * unit).sum((0, 1)))
        du = dy * s[name + "_weight"].float()
        outs.append((r * (du - unit * (du * unit).mean(-1, keepdim=True))).to(torch.bfloat16))
    return (*outs, *weights)


def _blocks(s, most):
    """(query rows, key rows, first and last query head, key head, rows of a strip) of every sequence and key head, for scores of at most `most` numbers at once."""
    case = s["case"]
    group = case["Hq"] // case["Hk"]
    q0 = k0 = 0
    for q, k in zip(*_lens(case)):
        for h in range(case["Hk"] if q > 0 else 0):
            yield slice(q0, q0 + q), slice(k0, k0 + k), slice(h * group, (h + 1) * group), h, max(1, min(q, most // max(1, group * k)))
        q0, k0 = q0 + q, k0 + k


def _plain_scores(q, k, first, rows, total, causal):
    """Weights of `rows` queries from `first` on out of `total`, all heads of a group, against all keys: softmax, 0 in rows that look at nothing."""
    x = torch.matmul(q, k.t()) * (k.shape[-1] ** -0.5)
    if causal:
        last = torch.arange(first, first + rows, device=q.device) + (k.shape[0] - total)
        x = x.masked_fill(torch.arange(k.shape[0], device=q.device)[None, :] > last[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total)


def _plain_attention(s, train):
    case = s["case"]
    out = torch.zeros_like(s["q"])
    if train:
        dq = torch.zeros(s["q"].shape, device="cuda")
        dk, dv = torch.zeros(s["k"].shape, device="cuda"), torch.zeros(s["v"].shape, device="cuda")
    for rows, keys, heads, h, strip in _blocks(s, 1 << 29):
        total = rows.stop - rows.start
        if keys.stop == keys.start:
            continue
        k, v = s["k"][keys, h].float(), s["v"][keys, h].float()
        for i in range(0, total, strip):
            n = min(strip, total - i)
            r = slice(rows.start + i, rows.start + i + n)
            q = s["q"][r, heads].float().transpose(0, 1)                      # heads of the group, queries, dimensions
            p = _plain_scores(q, k, i, n, total, case["causal"])
            o = torch.matmul(p, v)
            out[r, heads] = o.transpose(0, 1).to(torch.bfloat16)
            if train:
                do = s["dout"][r, heads].float().transpose(0, 1)
                dv[keys, h] += torch.matmul(p.transpose(1, 2), do).sum(0)
                dx = p * (torch.matmul(do, v.t()) - (do * o).sum(-1, keepdim=True)) * (k.shape[-1] ** -0.5)
                dq[r, heads] = torch.matmul(dx, k).transpose(0, 1)
                dk[keys, h] += torch.matmul(dx.transpose(1, 2), q).sum(0)
    if not train:
        return out
    return out, dq.to(torch.bfloat16), dk.to(torch.bfloat16), dv.to(torch.bfloat16)


def _slots(s, lens, before):
    """Page and place in the page of every token of the call."""
    page, place = [], []
    for b, (n, a) in enumerate(zip(lens, before)):
        t = torch.arange(a, a + n, device="cuda")
        page.append(s["table"][b, t // PAGE].long())
        place.append(t % PAGE)
    return torch.cat(page), torch.cat(place)


def _plain_store(s):
    case = s["case"]
    D, Hk = case["D"], case["Hk"]
    lens, before = _ints(case["q_lens"]), _ints(case["before"])
    page, place = _slots(s, lens, before)
    outs = []
    for name in ("k", "v"):
        words, scales = s["cache"][name + "_words"], s["cache"][name + "_scales"]
        step, low, n = quantise(s[name].float().view(-1, Hk, D // GROUP, GROUP))
        scales[page, :, place, :, 0] = step
        scales[page, :, place, :, 1] = low
        n = n.view(-1, Hk, D)
        if name == "k":
            words[page, :, place] = _k_words(n)
            got = _k_numbers(words[page, :, place])
        else:
            touched = page.unique()                                        # whole pages are taken apart and put together again
            numbers = _v_numbers(words[touched])
            at = torch.searchsorted(touched, page)
            numbers[at, :, place] = n
            words[touched] = _v_words(numbers)
            got = _v_numbers(words[touched])[at, :, place]
        pair = scales[page, :, place].float()
        outs.append((pair[..., 1:] + pair[..., :1] * got.view(-1, Hk, D // GROUP, GROUP)).view(-1, Hk, D).to(torch.bfloat16))
    return tuple(outs)


def _cached(s, b, n):
    """The first n keys and values of sequence b, (Hk, n, D) in 32 bits."""
    pages = s["table"][b, :-(-n // PAGE)].long()
    out = []
    for name, numbers in (("k", _k_numbers), ("v", _v_numbers)):
        pair = s["cache"][name + "_scales"][pages].float()
        x = numbers(s["cache"][name + "_words"][pages]).float()
        x = pair[..., 1:] + pair[..., :1] * x.view(*x.shape[:3], -1, GROUP)
        out.append(x.flatten(3).transpose(0, 1).flatten(1, 2)[:, :n])
    return out


def _plain_decode(s):
    case = s["case"]
    out = torch.zeros_like(s["q"])
    for b, n in enumerate(_ints(case["lens"])):
        if n == 0:
            continue
        k, v = _cached(s, b, n)
        q = s["q"][b].float().view(case["Hk"], -1, case["D"])
        x = torch.matmul(q, k.transpose(1, 2).contiguous()) * (case["D"] ** -0.5)
        p = torch.exp(x - x.amax(-1, keepdim=True))
        out[b] = (torch.matmul(p, v) / p.sum(-1, keepdim=True)).reshape(case["Hq"], case["D"]).to(torch.bfloat16)
    return out


# ---------------------------------------------------------------- one pass

def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if not own:
        if op == "norm":
            return _plain_norm(s)
        if op == "norm_back":
            return _plain_norm_back(s)
        if op in ("prompt", "train"):
            return _plain_attention(s, op == "train")
        return _plain_store(s) if op == "store" else _plain_decode(s)

    import paper_2508_20258_amd as swz
    if op == "norm":
        return swz.qk_norm_rope(s["q"], s["k"], s["q_weight"], s["k_weight"], s["cos"], s["sin"], s["positions"], eps=EPS, interleaved=case["interleaved"])
    if op == "norm_back":
        return swz.qk_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["cos"], s["sin"], s["positions"], eps=EPS,
                                         interleaved=case["interleaved"])
    if op == "prompt":
        return swz.attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=case["causal"])[0]
    if op == "train":
        out, lse = swz.attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=case["causal"])
        return (out, *swz.attention_backward(s["dout"], s["q"], s["k"], s["v"], out, lse, s["cu_q"], s["cu_k"], causal=case["causal"]))
    if op == "store":
        swz.cache4_append(s["cache"], s["k"], s["v"], s["cu_q"], s["before"], s["table"])
        return swz.cache4_read(s["cache"], s["cu_q"], s["before"], s["table"], s["k"].shape[0])
    return swz.cache4_attention(s["q"], s["cache"], s["lens"], s["table"], s["max_len"])


# ---------------------------------------------------------------- in 64 bits, from the definitions

def _exact_norm(s, op):
    T, h = s["positions"].shape[0], s["cos"].shape[1]
    D, inter = s["q"].shape[-1], s["case"]["interleaved"]
    first = torch.arange(h, device="cuda") * 2 if inter else torch.arange(h, device="cuda")
    second = first + (1 if inter else h)
    out, weights = [], []
    strip = max(1, (1 << 25) // (D * (s["q"].shape[1])))
    for name in ("q", "k"):
        x_all, w = s[name], s[name + "_weight"].double()
        res = torch.empty(x_all.shape, dtype=torch.float64, device="cuda")
        dw = torch.zeros(D, dtype=torch.float64, device="cuda")
        for i in range(0, T, strip):
            x = x_all[i:i + strip].double()
            at = s["positions"][i:i + strip].long()
            c, n = s["cos"][at].double().unsqueeze(1), s["sin"][at].double().unsqueeze(1)
            rms = ((x ** 2).sum(-1, keepdim=True) / D + EPS) ** 0.5
            if op == "norm":
                z = x / rms * w
                lo, hi = z[..., first], z[..., second]
                z[..., first], z[..., second] = lo * c - hi * n, hi * c + lo * n
                res[i:i + strip] = z
            else:
                g = s["d" + name][i:i + strip].double()
                lo, hi = g[..., first], g[..., second]
                g[..., first], g[..., second] = lo * c + hi * n, hi * c - lo * n
                dw += (g * x / rms).sum(1).sum(0)
                gw = g * w
                res[i:i + strip] = gw / rms - x * (gw * x).sum(-1, keepdim=True) / (D * rms ** 3)
        out.append(res)
        weights.append(dw)
    return tuple(out) if op == "norm" else (*out, *weights)


def _exact_attention(s, train):
    case = s["case"]
    group = case["Hq"] // case["Hk"]
    scale = case["D"] ** -0.5
    new = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    out = new(s["q"])
    dq, dk, dv = (new(s["q"]), new(s["k"]), new(s["v"])) if train else (None, None, None)
    q0 = k0 = 0
    for nq, nk in zip(*_lens(case)):
        strip = max(64, min(4096, (1 << 28) // max(1, nk)))
        for head in range(case["Hq"]):
            kh = head // group
            for i in range(0, nq, strip):
                n = min(strip, nq - i)
                seen = max(0, min(nk, nk - nq + i + n)) if case["causal"] else nk      # keys that any of these rows looks at
                if seen == 0:
                    continue
                r, c = slice(q0 + i, q0 + i + n), slice(k0, k0 + seen)
                q, k, v = s["q"][r, head].double(), s["k"][c, kh].double(), s["v"][c, kh].double()
                score = q @ k.t().contiguous() * scale
                if case["causal"]:
                    allowed = torch.ones((n, seen), dtype=torch.bool, device="cuda").tril(nk - nq + i)
                    score = torch.where(allowed, score, torch.full_like(score, -math.inf))
                weight = torch.nan_to_num((score - score.logsumexp(1, keepdim=True).nan_to_num(neginf=0.0)).exp(), nan=0.0)
                o = weight @ v
                out[r, head] = o
                if train:
                    do = s["dout"][r, head].double()
                    dv[c, kh] += weight.t().contiguous() @ do
                    ds = weight * (do @ v.t().contiguous() - (do * o).sum(1, keepdim=True))
                    dq[r, head] = ds @ k * scale
                    dk[c, kh] += ds.t().contiguous() @ q * scale
        q0, k0 = q0 + nq, k0 + nk
    return (out, dq, dk, dv) if train else out


def _exact_store(s):
    """The values that the format holds for these keys and values: of the 16 that low and step name, the one that the rounded quotient picks."""
    outs = []
    for name in ("k", "v"):
        x = s[name].double().unflatten(-1, (-1, GROUP))
        low, high = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
        step = ((high - low).float() / 15).to(torch.bfloat16).double()
        n = torch.where(step > 0, ((x - low).float() / step.float()).round().double(), 0.0).clamp(0, 15)
        outs.append((low + step * n).flatten(-2))
    return tuple(outs)


def _exact_decode(s):
    case = s["case"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    shifts = torch.tensor([4 * (i + 4 * h) for i in range(4) for h in range(2)], device="cuda", dtype=torch.int32)
    D, Hk = case["D"], case["Hk"]
    for b, n in enumerate(_ints(case["lens"])):
        if n == 0:
            continue
        pages = s["table"][b, :(n + PAGE - 1) // PAGE].long()
        for h in range(Hk):
            kw, vw = s["cache"]["k_words"][pages, h], s["cache"]["v_words"][pages, h]
            # dimension 32 a + 8 g + e of a key is number e of word (D / 32) g + a; token 8 o + e of a dimension is number e of word (o, dimension)
            k = torch.empty((len(pages), PAGE, D), dtype=torch.float64, device="cuda")
            v = torch.empty_like(k)
            for e in range(8):
                kn, vn = (kw >> shifts[e] & 15).double(), (vw >> shifts[e] & 15).double()
                for a in range(D // 32):
                    for g in range(4):
                        k[..., 32 * a + 8 * g + e] = kn[..., D // 32 * g + a]
                v[:, e::8] = vn
            for x, name in ((k, "k_scales"), (v, "v_scales")):
                pair = s["cache"][name][pages, h].double().repeat_interleave(GROUP, 2)
                x.mul_(pair[..., 0]).add_(pair[..., 1])
            heads = slice(h * (case["Hq"] // Hk), (h + 1) * (case["Hq"] // Hk))
            score = s["q"][b, heads].double() @ k.flatten(0, 1)[:n].t().contiguous() * D ** -0.5
            out[b, heads] = score.softmax(1) @ v.flatten(0, 1)[:n]
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("norm", "norm_back"):
        return _exact_norm(s, op)
    if op in ("prompt", "train"):
        return _exact_attention(s, op == "train")
    return _exact_store(s) if op == "store" else _exact_decode(s)
