"""A step with drafted tokens over a cache in bfloat16, as its operators are measured on one MI355X: keys and values appended to the cache with the rotation of
queries and keys on the way, attention of the drafted tokens over it, the verification of the drafts, and the accepted path's keys and values kept.

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes what a program has in hand before the call, `run()` is one pass, `work()` its
minimal traffic and arithmetic, `exact()` the same result in 64 bits.  With `own` false `run()` computes the plain form from elementary torch operations, with `own`
true it calls the package.

The tokens of all sequences are packed: `cu` holds their first tokens and the total.  A sequence's tokens are a tree: token 0, the root, is the last one that stands, the
others are drafts, and in a case of `branch` B the parent of token i is (i - 1) // B: a chain where B is 1.  The cache is pages of (k_heads, page_tokens, head_dim).
"""
import math
import random

import torch

own = False

# what a drawn case costs at most, no more than the largest listed one of its kind
MAX_APPEND = 32768 * 48 * 128                # elements of queries, keys and values
MAX_KEYS = 131072 * 8 * 128                  # of K in the cache
MAX_PRODUCT = 131072 * 64 * 32 * 128         # pairs of a query and a key, times heads and their size
MAX_PROBS = 64 * 6 * 128000                  # probabilities of a kind
MAX_KEPT = 128 * 64 * 8 * 128


def listed():
    return [
        # a step's tokens into the cache: 16 sequences with trees of 8; the launch is most of it
        dict(name="append_step", op="append", Hq=32, Hk=8, D=128, R=128, interleaved=False, page=64, branch=2, lens=_text([8] * 16), before=_text(_ragged(3, 16, 1, 1000))),
        # whole prompts, and next pieces of prompts, positions as they follow each other
        dict(name="append_prompt", op="append", Hq=32, Hk=8, D=128, R=128, interleaved=False, page=64, branch=1, lens="16384,8192,5000,2047,1,0,1144", before="0,0,100,7,63,0,4096"),
        # small heads of which half is turned, in pairs of neighbours, small pages, trees of all sizes
        dict(name="append_64", op="append", Hq=16, Hk=16, D=64, R=32, interleaved=True, page=16, branch=3, lens=_text(_ragged(4, 77, 1, 64) + [0]), before=_text(_ragged(5, 78, 1, 500))),
        # single tokens over a few short sequences, where latency counts
        dict(name="attend_tokens", op="attend", Hq=32, Hk=8, D=128, page=64, branch=1, nodes="1,1,1,1,1,1", lens="1000,512,1,0,77,2048"),
        # a batch of trees over contexts of all lengths
        dict(name="attend_batch", op="attend", Hq=32, Hk=8, D=128, page=64, branch=2, nodes=_text([32] * 32), lens=_text(_ragged(6, 31, 512, 8192) + [8192])),
        # one long context, the largest tree, eight query heads to a key head
        dict(name="attend_long", op="attend", Hq=32, Hk=4, D=128, page=128, branch=4, nodes="64", lens="131072"),
        # small heads in small pages, trees of all sizes, one without tokens, one without a context
        dict(name="attend_64", op="attend", Hq=16, Hk=8, D=64, page=16, branch=3, nodes=_text(_ragged(7, 30, 1, 64) + [0, 7]), lens=_text(_ragged(8, 31, 100, 10000) + [7])),
        # chains of five drafts that were drawn from the draft's probabilities, a full batch
        dict(name="verify_chains", op="verify", V=128000, half=False, drawn=True, branch=1, nodes=_text([6] * 64)),
        # trees of the likeliest tokens, of all sizes, probabilities as a softmax in bfloat16 leaves them
        dict(name="verify_trees", op="verify", V=32000, half=True, drawn=False, branch=3, nodes=_text(_ragged(9, 15, 1, 64) + [64])),
        # trees whose children were drawn from the draft's probabilities, a vocabulary that is no multiple of anything
        dict(name="verify_drawn", op="verify", V=50257, half=False, drawn=True, branch=3, nodes="13,20,1,13,40,13,7,13"),
        # the block appended and its accepted path kept: a few sequences, and a full batch of large trees
        dict(name="keep_step", op="keep", Hk=8, D=128, page=64, branch=2, lens=_text([16] * 16), before=_text(_ragged(10, 16, 1, 1000))),
        dict(name="keep_batch", op="keep", Hk=8, D=128, page=32, branch=1, lens=_text([64] * 128), before=_text(_ragged(11, 128, 1, 300))),
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


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "verify", "verify", "keep"])
    while True:
        D, page, branch = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128, 256]), rng.choice([1, 1, 2, 3, 5])
        Hk = rng.choice([1, 2, 4, 8, 16])
        Hq = Hk * rng.choice([g for g in (1, 2, 3, 4, 5, 8, 16) if g * Hk <= 64])
        n = _log_int(rng, 1, 128)
        nodes = [_log_int(rng, 1, rng.choice([8, 64])) for _ in range(n)]
        if op == "append":
            lens = [_log_int(rng, 1, 32768) for _ in range(n)] if branch == 1 else nodes
            if sum(lens) * (Hq + 2 * Hk) * D <= MAX_APPEND:
                return dict(op=op, Hq=Hq, Hk=Hk, D=D, R=rng.choice([D, D, D // 2, 16]), interleaved=rng.random() < 0.3, page=page, branch=branch, lens=_text(lens),
                            before=_text([rng.choice([0, _log_int(rng, 1, 1000)]) for _ in lens]))
        if op == "attend":
            longest = _log_int(rng, 16, 131072)
            lens = [k if rng.random() < 0.05 else k + q for q, k in zip(nodes, (_log_int(rng, 1, longest) for _ in nodes))]
            if sum(lens) * Hk * D <= MAX_KEYS and sum(q * k for q, k in zip(nodes, lens)) * Hq * D <= MAX_PRODUCT:
                return dict(op=op, Hq=Hq, Hk=Hk, D=D, page=page, branch=branch, nodes=_text(nodes), lens=_text(lens))
        if op == "verify":
            V = _log_int(rng, 500, 200000)
            if sum(nodes) * V <= MAX_PROBS:
                return dict(op=op, V=V, half=rng.random() < 0.4, drawn=rng.random() < 0.5, branch=branch, nodes=_text(nodes))
        if op == "keep" and sum(nodes) * Hk * D <= MAX_KEPT:
            return dict(op=op, Hk=Hk, D=D, page=page, branch=branch, lens=_text(nodes), before=_text([rng.choice([0, _log_int(rng, 1, 500)]) for _ in nodes]))


def _parents(n, branch):
    return [max(0, (i - 1) // branch) for i in range(n)]


def _depths(n, branch):
    out = []
    for i, p in enumerate(_parents(n, branch)):
        out.append(out[p] + 1 if i else 0)
    return out


def _masks(n, branch):
    """For each token of a tree the bits of those on its path, its own among them, as signed 64-bit numbers."""
    out = []
    for i, p in enumerate(_parents(n, branch)):
        out.append(1 << i | (out[p] if i else 0))
    return [m - (1 << 64) if m >> 63 else m for m in out]


def _attend_pairs(case):
    pairs = 0
    for n, length in zip(_ints(case["nodes"]), _ints(case["lens"])):
        context = length - n
        # of a block that is cut at its front (fewer positions than tokens) only the last ones are there
        pairs += n * context + sum(d + 1 for d in _depths(n, case["branch"])) if context >= 0 else length
    return pairs


def work(case):
    op = case["op"]
    if op == "append":
        n, D, Hq, Hk = sum(_ints(case["lens"])), case["D"], case["Hq"], case["Hk"]
        return {"bytes": n * (4 * D * (Hq + 2 * Hk) + 4 * case["R"]), "flops": 3 * n * case["R"] * (Hq + Hk)}
    if op == "attend":
        D, n = case["D"], sum(_ints(case["nodes"]))
        return {"bytes": 4 * D * case["Hk"] * sum(_ints(case["lens"])) + 4 * D * case["Hq"] * n, "flops": 4 * D * case["Hq"] * _attend_pairs(case)}
    if op == "verify":
        # the row that the new token is drawn from, of both where the drafts were drawn, and a value of each node on the way
        rows = sum(1 for n in _ints(case["nodes"]) if n > 0) * (2 if case["drawn"] else 1)
        return {"bytes": rows * case["V"] * (2 if case["half"] else 4) + 16 * sum(_ints(case["nodes"])), "flops": 2 * rows * case["V"]}
    n = sum(_ints(case["lens"]))
    return {"bytes": n * 8 * case["D"] * case["Hk"], "flops": 0}


# ---------------------------------------------------------------- inputs

def _normal(g, shape, scale=1.0):
    """bfloat16 normal values, made in strips: the 32-bit values of a large tensor need not exist at once."""
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, device="cuda", generator=g) * scale
    return out


def _device_ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _cu(lens):
    return torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)


def _table(g, lens, page):
    """Pages of each sequence, in no order; entries past a sequence's end are -1."""
    need = [-(-n // page) for n in lens]
    order = torch.randperm(max(1, sum(need)), device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(lens), max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    first = 0
    for b, n in enumerate(need):
        table[b, :n] = order[first:first + n]
        first += n
    return table, max(1, sum(need))


def _angles(R):
    angle = torch.arange(40000, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(0, R, 2, device="cuda").double() / R)
    return angle.cos().float(), angle.sin().float()


def _probs(g, rows, V, half):
    """Rows of a target's probabilities and of a draft's that is near it."""
    type_ = torch.bfloat16 if half else torch.float32
    out = [torch.empty((rows, V), dtype=type_, device="cuda") for _ in range(2)]
    strip = max(1, (1 << 26) // V)
    for i in range(0, rows, strip):
        n = min(strip, rows - i)
        x = torch.randn((n, V), device="cuda", generator=g) * 2.5
        out[0][i:i + n] = x.softmax(1)
        out[1][i:i + n] = (x + 0.8 * torch.randn((n, V), device="cuda", generator=g)).softmax(1)
    return out


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = dict(case=case)
    if op in ("append", "keep"):
        lens, before, D, Hk = _ints(case["lens"]), _ints(case["before"]), case["D"], case["Hk"]
        n, Hq = sum(lens), case.get("Hq", 0)
        rows = _normal(g, (n, (Hq + 2 * Hk) * D))                        # the rows that a projection writes
        if Hq:
            s["q"] = rows[:, :Hq * D].view(n, Hq, D)
        s["k"] = rows[:, Hq * D:(Hq + Hk) * D].view(n, Hk, D)
        s["v"] = rows[:, (Hq + Hk) * D:].view(n, Hk, D)
        s["cu"], s["before"] = _cu(lens), _device_ints(before)
        s["table"], pages = _table(g, [a + b for a, b in zip(lens, before)], case["page"])
        s["cache"] = [torch.zeros((pages, Hk, case["page"], D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        if op == "append":
            s["cos"], s["sin"] = _angles(case["R"])
            s["positions"] = None
            if case["branch"] > 1:
                s["positions"] = _device_ints([b + d for b, m in zip(before, lens) for d in _depths(m, case["branch"])])
        else:
            # a path from the root downwards, as long as chance has it
            rng = random.Random(seed)
            path, accepted = [], []
            for m in lens:
                at, mine = 0, [0]
                while m > 0 and rng.random() < 0.8:
                    children = [c for c in range(at * case["branch"] + 1, (at + 1) * case["branch"] + 1) if c < m]
                    if not children:
                        break
                    at = rng.choice(children)
                    mine.append(at)
                accepted.append(len(mine) - 1 if m else 0)
                path += (mine + [-1] * m)[:m]
            s["path"], s["accepted"] = _device_ints(path), _device_ints(accepted)
    elif op == "attend":
        nodes, lens, D, Hk = _ints(case["nodes"]), _ints(case["lens"]), case["D"], case["Hk"]
        s["table"], pages = _table(g, lens, case["page"])
        s["cache"] = [_normal(g, (pages, Hk, case["page"], D)) for _ in range(2)]
        s["q"] = _normal(g, (sum(nodes), case["Hq"], D), 1.5)            # scores of a spread of 1.5
        s["cu"], s["lengths"], s["longest"] = _cu(nodes), _device_ints(lens), max(lens)
        s["tree"] = None
        if case["branch"] > 1:
            s["tree"] = _device_ints([m for n in nodes for m in _masks(n, case["branch"])], torch.int64)
    else:
        nodes, branch = _ints(case["nodes"]), case["branch"]
        n = sum(nodes)
        s["target"], s["draft"] = _probs(g, n, case["V"], case["half"])
        s["cu"] = _cu(nodes)
        s["uniforms"] = torch.rand(n, device="cuda", generator=g)
        first = [sum(nodes[:b]) for b in range(len(nodes))]
        row = _device_ints([f + p for f, m in zip(first, nodes) for p in _parents(m, branch)], torch.int64)      # of each node's parent
        child = _device_ints([(i - 1) % branch if i else 0 for m in nodes for i in range(m)], torch.int64)
        if case["drawn"]:
            picks = []
            for i in range(0, n, 64):
                picks.append(torch.multinomial(s["draft"][row[i:i + 64]].float(), 1, generator=g)[:, 0])
            s["tokens"] = torch.cat(picks).to(torch.int32)
        else:
            top = s["draft"].float().topk(branch, dim=1).indices
            s["tokens"] = top[row, child].to(torch.int32)
            s["draft"] = None
        s["parents"] = None if branch == 1 else _device_ints([p for m in nodes for p in _parents(m, branch)])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and "cache" in s:
        import paper_2508_20258_amd as swz
        s["cache"] = swz.Cache16(*s["cache"])
    return s


# ---------------------------------------------------------------- the plain forms

def _turn(x, c, s, interleaved):
    """x (T, H, D), 32-bit: the pairs of its first R dimensions turned; c, s (T, R / 2)."""
    h = c.shape[-1]
    a, b = (x[..., 0:2 * h:2], x[..., 1:2 * h:2]) if interleaved else (x[..., :h], x[..., h:2 * h])
    c, s = c[:, None], s[:, None]
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., 2 * h:]), -1)


def _places(s):
    """Page, place in the page, and position of every token of the call."""
    case, page = s["case"], s["case"]["page"]
    at = [torch.arange(a, a + n, device="cuda") for n, a in zip(_ints(case["lens"]), _ints(case["before"]))]
    pages = [s["table"][b, t // page].long() for b, t in enumerate(at)]
    at = torch.cat(at)
    return torch.cat(pages), at % page, at


def _plain_append(s, turned=True):
    page, place, at = _places(s)
    k, q = s["k"], None
    if turned:
        at = at if s["positions"] is None else s["positions"].long()
        c, n = s["cos"][at], s["sin"][at]
        q, k = (_turn(x.float(), c, n, s["case"]["interleaved"]).to(torch.bfloat16) for x in (s["q"], k))
    s["cache"][0][page, :, place] = k
    s["cache"][1][page, :, place] = s["v"]
    return (q, *s["cache"]) if turned else tuple(s["cache"])


def _plain_keep(s):
    case, page = s["case"], s["case"]["page"]
    _plain_append(s, False)
    # in rising order, all sequences at once: a place is read before it is written
    first, before = s["cu"][:-1].long(), s["before"].long()
    rows = torch.arange(len(before), device="cuda")
    for i in range(1, max(_ints(case["lens"]))):
        here = (i <= s["accepted"]).nonzero()[:, 0]
        source = before[here] + s["path"][first[here] + i].long()
        to = before[here] + i
        a, b = s["table"][rows[here], source // page].long(), s["table"][rows[here], to // page].long()
        for x in s["cache"]:
            x[b, :, to % page] = x[a, :, source % page]
    return tuple(s["cache"])


def _plain_attend(s):
    case, page = s["case"], s["case"]["page"]
    Hk, D = case["Hk"], case["D"]
    out = torch.zeros_like(s["q"])
    first = 0
    for b, (n, length) in enumerate(zip(_ints(case["nodes"]), _ints(case["lens"]))):
        rows = slice(first, first + n)
        first += n
        if n == 0 or length == 0:
            continue
        pages = s["table"][b, :-(-length // page)].long()
        at, token = torch.arange(length, device="cuda") - (length - n), torch.arange(n, device="cuda")
        if s["tree"] is None:
            seen = at[None, :] <= token[:, None]
        else:
            seen = (at < 0)[None, :] | (s["tree"][rows][:, None] >> at.clamp(min=0)[None, :] & 1).bool()
        for h in range(Hk):
            k, v = (x[pages, h].flatten(0, 1)[:length].float() for x in s["cache"])
            q = s["q"][rows, h * (case["Hq"] // Hk):(h + 1) * (case["Hq"] // Hk)].float().transpose(0, 1)
            x = (torch.matmul(q, k.t()) * D ** -0.5).masked_fill(~seen, -math.inf)
            top = x.amax(-1, keepdim=True)
            p = torch.exp(x - torch.where(torch.isinf(top), torch.zeros_like(top), top))
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
            out[rows, h * (case["Hq"] // Hk):(h + 1) * (case["Hq"] // Hk)] = o.transpose(0, 1).to(torch.bfloat16)
    return out


def _plain_verify(s):
    """All sequences at once, node by node; what is left of the target's probabilities in 64 bits."""
    case = s["case"]
    nodes = _ints(case["nodes"])
    B = len(nodes)
    first = s["cu"][:-1].long()
    count = s["cu"][1:].long() - first
    rows = torch.arange(B, device="cuda")
    cur, accepted = torch.zeros_like(first), torch.zeros_like(first)
    path = torch.full((sum(nodes),), -1, dtype=torch.int32, device="cuda")
    path[first[count > 0]] = 0
    left = s["target"][first.clamp(max=max(0, sum(nodes) - 1))].double()
    mass = torch.ones(B, dtype=torch.float64, device="cuda")
    for i in range(1, max(nodes)):
        at = (first + i).clamp(max=sum(nodes) - 1)
        parent = torch.full_like(first, i - 1) if s["parents"] is None else s["parents"][at].long()
        tested = (i < count) & (parent == cur)
        x, u = s["tokens"][at].long(), s["uniforms"][at].double()
        mine = left[rows, x]
        if s["draft"] is None:
            good = tested & (mine > (u * mass).clamp(min=0))
            bad = tested & ~good
            mass = mass - torch.where(bad, mine, torch.zeros_like(mine))
            left[rows, x] = torch.where(bad, torch.zeros_like(mine), mine)
        else:
            q = s["draft"][first + cur].double()
            good = tested & (u * q[rows, x] < mine)
            bad = tested & ~good
            less = (left - q).clamp(min=0)
            total = less.sum(1, keepdim=True)
            left = torch.where(bad[:, None] & (total > 0), less / total, left)
        cur = torch.where(good, torch.full_like(cur, i), cur)
        accepted = accepted + good
        path[(first + accepted)[good]] = i
        left = torch.where(good[:, None], s["target"][first.clamp(max=sum(nodes) - 1) + torch.where(good, cur, torch.zeros_like(cur))].double(), left)
        mass = torch.where(good, torch.ones_like(mass), mass)
    total = left.cumsum(1)
    r = s["uniforms"][first.clamp(max=sum(nodes) - 1)].double() * total[:, -1]
    token = torch.searchsorted(total, r[:, None], right=True)[:, 0]
    return accepted.to(torch.int32), path, torch.where(count > 0, token, torch.full_like(token, -1)).to(torch.int32)


# ---------------------------------------------------------------- one pass

def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "verify": _plain_verify, "keep": _plain_keep}[op](s)

    import paper_2508_20258_amd as swz
    if op == "append":
        q = swz.cache16_append(s["cache"], s["k"], s["v"], s["cu"], s["before"], s["table"], q=s["q"], cos=s["cos"], sin=s["sin"], positions=s["positions"],
                               interleaved=case["interleaved"])
        return (q, *s["cache"])
    if op == "attend":
        return swz.cache16_attention(s["q"], s["cache"], s["cu"], s["lengths"], s["table"], tree=s["tree"], max_length=s["longest"])
    if op == "verify":
        return swz.verify_drafts(s["target"], s["tokens"], s["cu"], s["uniforms"], draft_probs=s["draft"], parents=s["parents"])
    swz.cache16_append(s["cache"], s["k"], s["v"], s["cu"], s["before"], s["table"])
    swz.cache16_keep(s["cache"], s["cu"], s["before"], s["path"], s["accepted"], s["table"])
    return tuple(s["cache"])


# ---------------------------------------------------------------- in 64 bits, from the definitions

def _exact_append(s):
    case = s["case"]
    page, R = case["page"], case["R"]
    pair = torch.arange(R // 2, device="cuda")
    lo = 2 * pair if case["interleaved"] else pair
    hi = lo + (1 if case["interleaved"] else R // 2)
    q = s["q"].double()
    cache = [torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in s["cache"]]
    first = 0
    for b, (n, a) in enumerate(zip(_ints(case["lens"]), _ints(case["before"]))):
        rows = slice(first, first + n)
        first += n
        at = torch.arange(a, a + n, device="cuda")
        angle = at if s["positions"] is None else s["positions"][rows].long()
        c, sn = s["cos"].double()[angle].unsqueeze(1), s["sin"].double()[angle].unsqueeze(1)
        k = s["k"][rows].double()
        for x in (q[rows], k):
            y, z = x[..., lo], x[..., hi]
            x[..., lo], x[..., hi] = y * c - z * sn, z * c + y * sn
        where = s["table"][b].long()[at.div(page, rounding_mode="floor")]
        cache[0][where, :, at.remainder(page)] = k
        cache[1][where, :, at.remainder(page)] = s["v"][rows].double()
    return (q, *cache)


def _exact_keep(s):
    case = s["case"]
    page, first = case["page"], 0
    cache = [torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in s["cache"]]
    path, accepted = s["path"].tolist(), s["accepted"].tolist()
    for b, (n, a) in enumerate(zip(_ints(case["lens"]), _ints(case["before"]))):
        # which token of the block ends up at each of its places
        held = list(range(n))
        held[:accepted[b] + 1] = path[first:first + accepted[b] + 1] if n else []
        at = torch.arange(a, a + n, device="cuda")
        where = s["table"][b].long()[at.div(page, rounding_mode="floor")]
        rows = torch.tensor([first + i for i in held], dtype=torch.int64, device="cuda")
        for x, new in zip(cache, (s["k"], s["v"])):
            x[where, :, at.remainder(page)] = new[rows].double()
        first += n
    return tuple(cache)


def _exact_attend(s):
    case = s["case"]
    page, group = case["page"], case["Hq"] // case["Hk"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, length) in enumerate(zip(_ints(case["nodes"]), _ints(case["lens"]))):
        base = length - n
        allowed = torch.ones((n, length), dtype=torch.bool)
        for i, mask in enumerate(_masks(n, case["branch"])):
            for j in range(n):
                if base + j >= 0:
                    allowed[i, base + j] = bool(mask >> j & 1)
        allowed = allowed.cuda()
        for head in range(case["Hq"] if n and length else 0):
            pages = s["table"][b, :(length + page - 1) // page].long()
            k, v = (x[pages, head // group].reshape(-1, case["D"])[:length].double() for x in s["cache"])
            score = s["q"][first:first + n, head].double() @ k.t().contiguous() / math.sqrt(case["D"])
            score = torch.where(allowed, score, torch.full_like(score, -math.inf))
            weight = torch.nan_to_num((score - score.logsumexp(1, keepdim=True).nan_to_num(neginf=0.0)).exp(), nan=0.0)
            out[first:first + n, head] = weight @ v
        first += n
    return out


def _exact_verify(s):
    """Sequence by sequence, as the rule reads."""
    case = s["case"]
    tokens, uniforms, branch = s["tokens"].tolist(), s["uniforms"].tolist(), case["branch"]
    accepted, path, new = [], [], []
    first = 0
    for n in _ints(case["nodes"]):
        if n == 0:
            accepted.append(0)
            new.append(-1)
            continue
        way = [0]
        while True:
            row = first + way[-1]
            p = s["target"][row].double()
            mass = 1.0
            chosen = None
            for c in range(way[-1] * branch + 1, min(n, (way[-1] + 1) * branch + 1)):
                x, u = tokens[first + c], uniforms[first + c]
                if s["draft"] is None:
                    if float(p[x]) > max(u * mass, 0.0):
                        chosen = c
                        break
                    mass -= float(p[x])
                    p[x] = 0.0
                else:
                    q = s["draft"][row].double()
                    if u * float(q[x]) < float(p[x]):
                        chosen = c
                        break
                    rest = torch.relu(p - q)
                    total = rest.sum()
                    if float(total) > 0:
                        p = rest / total
            if chosen is None:
                break
            way.append(chosen)
        sums = torch.cumsum(p, 0)
        new.append(int((sums <= uniforms[first] * sums[-1]).sum()))
        accepted.append(len(way) - 1)
        path += way + [-1] * (n - len(way))
        first += n
    return tuple(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (accepted, path, new))


def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "verify": _exact_verify, "keep": _exact_keep}[case["op"]](s)
