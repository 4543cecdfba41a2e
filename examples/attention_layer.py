"""An attention layer made of the library's operators, as a training step and as a server would run it.

The layer: rows = x @ w_in, of which queries, keys and values are views; norm and rotation of queries and keys; causal attention; out @ w_out.

    python examples/attention_layer.py        # on the GPU: both paths, their errors and times
"""
from __future__ import annotations

import os
import sys
import time
from typing import NamedTuple

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2508_20258_amd as swz  # noqa: E402


class Layer(NamedTuple):
    w_in: torch.Tensor           # (width, (q_heads + 2 k_heads) * head_dim)
    w_out: torch.Tensor          # (q_heads * head_dim, width)
    q_weight: torch.Tensor       # (head_dim,)
    k_weight: torch.Tensor
    cos: torch.Tensor            # (positions, rotary_dim / 2)
    sin: torch.Tensor
    q_heads: int
    k_heads: int

    @property
    def head_dim(self) -> int:
        return self.q_weight.shape[0]


class Saved(NamedTuple):         # what the backward pass needs of the forward pass
    x: torch.Tensor
    rows: torch.Tensor
    q: torch.Tensor
    k: torch.Tensor
    out: torch.Tensor
    lse: torch.Tensor
    cu: torch.Tensor
    positions: torch.Tensor


def make_layer(width: int, q_heads: int, k_heads: int, head_dim: int, positions: int, seed: int = 0, device: str = "cuda") -> Layer:
    g = torch.Generator().manual_seed(seed)

    def randn(*shape, scale):
        return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16).to(device)

    angles = torch.arange(positions)[:, None] * 10000.0 ** (-torch.arange(head_dim // 2) / (head_dim // 2))
    return Layer(randn(width, (q_heads + 2 * k_heads) * head_dim, scale=width ** -0.5), randn(q_heads * head_dim, width, scale=(q_heads * head_dim) ** -0.5),
                 1 + randn(head_dim, scale=0.1), 1 + randn(head_dim, scale=0.1), angles.cos().float().to(device), angles.sin().float().to(device), q_heads, k_heads)


def heads_of(rows, layer: Layer):
    """Queries, keys and values where they stand in rows of all of them: no copies."""
    n, d = rows.shape[0], layer.head_dim
    sizes = [layer.q_heads * d, layer.k_heads * d, layer.k_heads * d]
    return [t.view(n, -1, d) for t in rows.split(sizes, 1)]


def project(x, layer: Layer, positions):
    """Rows of the projection, and queries and keys normed and turned."""
    rows = swz.gemm(x, layer.w_in)
    q, k, v = heads_of(rows, layer)
    return rows, *swz.qk_norm_rope(q, k, layer.q_weight, layer.k_weight, layer.cos, layer.sin, positions), v


def forward(layer: Layer, x, cu, positions):
    """x: a multiple of 8 tokens, as the transposes of the backward pass want it.  What stands behind the last sequence is padding, whose outputs and gradients are 0."""
    rows, q, k, v = project(x, layer, positions)
    out, lse = swz.attention(q, k, v, cu, out=torch.zeros_like(q))
    return swz.gemm(out.view(x.shape[0], -1), layer.w_out), Saved(x, rows, q, k, out, lse, cu, positions)


def backward(layer: Layer, dy, s: Saved):
    """Gradients of x and of the four weights."""
    n = dy.shape[0]
    q_in, k_in, v = heads_of(s.rows, layer)
    dw_out = swz.gemm(swz.transpose(s.out.view(n, -1)), dy)
    dout = swz.gemm(dy, swz.transpose(layer.w_out)).view(s.out.shape)
    drows = torch.zeros_like(s.rows)                       # the gradients of queries, keys and values go where the projection's gradient wants them
    dq, dk, dv = heads_of(drows, layer)
    swz.attention_backward(dout, s.q, s.k, v, s.out, s.lse, s.cu, None, dq, dk, dv)
    _, _, dq_weight, dk_weight = swz.qk_norm_rope_backward(dq, dk, q_in, k_in, layer.q_weight, layer.k_weight, layer.cos, layer.sin, s.positions, dq, dk)
    return swz.gemm(drows, swz.transpose(layer.w_in)), swz.gemm(swz.transpose(s.x), drows), dw_out, dq_weight, dk_weight


class Server:
    """Sequences whose keys and values stay in a 4-bit cache.  Pages are handed out in turn as sequences grow."""

    def __init__(self, layer: Layer, sequences: int, longest: int, page_tokens: int = 64):
        per = -(-longest // page_tokens)
        self.layer, self.longest = layer, longest
        self.cache = swz.kv_cache4(sequences * per, layer.k_heads, layer.head_dim, page_tokens)
        order = torch.randperm(sequences * per, generator=torch.Generator().manual_seed(1))        # any order will do
        self.table = order.view(sequences, per).to(torch.int32).cuda()
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device="cuda")

    def prompt(self, x, counts):
        """The next counts[b] tokens of every sequence, packed: their keys and values into the cache, and attention over all that the cache holds."""
        n = x.shape[0]
        cu = torch.tensor([0, *counts], device="cuda").cumsum(0).to(torch.int32)
        before = self.lengths
        of = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), torch.tensor(counts, device="cuda"))
        positions = (torch.arange(n, device="cuda") - cu[of] + before[of]).to(torch.int32)
        _, q, k, v = project(x, self.layer, positions)
        swz.cache4_append(self.cache, k, v, cu, before, self.table)
        self.lengths = before + torch.tensor(counts, dtype=torch.int32, device="cuda")
        held = self.lengths.tolist()
        if held == list(counts):                           # nothing was there before: the new keys and values are all
            out, _ = swz.attention(q, k, v, cu)
        else:
            cu_k = torch.tensor([0, *held], device="cuda").cumsum(0).to(torch.int32)
            k, v = swz.cache4_read(self.cache, cu_k, torch.zeros_like(before), self.table, sum(held))
            out, _ = swz.attention(q, k, v, cu, cu_k)
        return swz.gemm(out.view(n, -1), self.layer.w_out)

    def token(self, x):
        """One token of every sequence."""
        n = x.shape[0]
        _, q, k, v = project(x, self.layer, self.lengths)
        swz.cache4_append(self.cache, k, v, torch.arange(n + 1, dtype=torch.int32, device="cuda"), self.lengths, self.table)
        self.lengths = self.lengths + 1
        out = swz.cache4_attention(q, self.cache, self.lengths, self.table, self.longest)
        return swz.gemm(out.view(n, -1), self.layer.w_out)


def plain(layer: Layer, x, cu, positions):
    """The layer in float32 on the CPU, for autograd and comparison."""
    n, d = x.shape[0], layer.head_dim
    q, k, v = heads_of(x @ layer.w_in, layer)
    c, s = layer.cos[positions][:, None], layer.sin[positions][:, None]

    def norm_turn(t, w):
        t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6) * w
        a, b = t.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    q, k = norm_turn(q, layer.q_weight), norm_turn(k, layer.k_weight)
    outs = []
    for lo, hi in zip(cu, cu[1:]):
        m = hi - lo
        group = layer.q_heads // layer.k_heads
        kk, vv = k[lo:hi].repeat_interleave(group, 1).transpose(0, 1), v[lo:hi].repeat_interleave(group, 1).transpose(0, 1)
        scores = (q[lo:hi].transpose(0, 1) @ kk.transpose(1, 2) * d ** -0.5).masked_fill(torch.ones(m, m).triu(1).bool(), float("-inf"))
        outs.append((scores.softmax(-1) @ vv).transpose(0, 1).reshape(m, -1))
    return torch.cat(outs) @ layer.w_out


def error(got, want) -> float:
    return float((got.double().cpu() - want.double()).norm() / want.double().norm())


def train(lens=(700, 1, 333), width=512, q_heads=8, k_heads=2, head_dim=128):
    """One step, and how far its results are from float32 with autograd: relative errors by name."""
    layer = make_layer(width, q_heads, k_heads, head_dim, max(lens))
    n, g = sum(lens), torch.Generator().manual_seed(5)
    padding = -n % 8
    x, dy = (torch.cat([torch.randn(n, width, generator=g), torch.zeros(padding, width)]).to(torch.bfloat16).cuda() for _ in range(2))
    cu = torch.tensor([0, *lens]).cumsum(0)
    positions = torch.cat([*(torch.arange(m) for m in lens), torch.zeros(padding, dtype=torch.int64)])
    y, saved = forward(layer, x, cu.to(torch.int32).cuda(), positions.to(torch.int32).cuda())
    grads = backward(layer, dy, saved)
    f = [t.float().cpu().requires_grad_() if isinstance(t, torch.Tensor) else t for t in layer]
    xf = x[:n].float().cpu().requires_grad_()
    yf = plain(Layer(*f), xf, cu.tolist(), positions[:n])
    yf.backward(dy[:n].float().cpu())
    names = ("x", "w_in", "w_out", "q_weight", "k_weight")
    assert not y[n:].any() and not grads[0][n:].any()
    return {"y": error(y[:n], yf.detach()), **{"d" + m: error(a, b.grad) for m, a, b in zip(names, (grads[0][:n], *grads[1:]), (xf, *f[:4]))}}


def serve(lens=(300, 37, 512), tokens=8, width=512, q_heads=8, k_heads=2, head_dim=128):
    """Prompts in two pieces, then single tokens: relative errors of each path against float32 without a cache."""
    total = [m + tokens for m in lens]
    layer = make_layer(width, q_heads, k_heads, head_dim, max(total))
    xs = [torch.randn(m, width, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16) for i, m in enumerate(total)]
    f = Layer(*(t.float().cpu() if isinstance(t, torch.Tensor) else t for t in layer))
    want = [plain(f, x.float(), [0, len(x)], torch.arange(len(x))) for x in xs]
    server, first = Server(layer, len(lens), max(total)), [m // 2 for m in lens]
    a = server.prompt(torch.cat([x[:m] for x, m in zip(xs, first)]).cuda(), first)
    b = server.prompt(torch.cat([x[m:e] for x, m, e in zip(xs, first, lens)]).cuda(), [e - m for m, e in zip(first, lens)])
    steps = [server.token(torch.stack([x[e + i] for x, e in zip(xs, lens)]).cuda()) for i in range(tokens)]
    return {"first piece": error(a, torch.cat([w[:m] for w, m in zip(want, first)])),
            "second piece": error(b, torch.cat([w[m:e] for w, m, e in zip(want, first, lens)])),
            "single tokens": error(torch.stack(steps), torch.stack([torch.stack([w[e + i] for w, e in zip(want, lens)]) for i in range(tokens)]))}


def seconds(f, repeat: int = 10) -> float:
    for _ in range(2):
        f()
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(repeat):
        f()
    torch.cuda.synchronize()
    return (time.perf_counter() - start) / repeat


def main() -> None:
    for name, e in (("training step", train()), ("serving", serve())):
        print(name + ", relative errors: " + ", ".join(f"{k} {v:.4f}" for k, v in e.items()), flush=True)
    layer = make_layer(4096, 32, 8, 128, 8192)
    x = torch.randn(8192, 4096, device="cuda").to(torch.bfloat16)
    cu, positions = torch.tensor([0, 4096, 8192], dtype=torch.int32, device="cuda"), torch.arange(4096, dtype=torch.int32, device="cuda").repeat(2)

    def step():
        y, saved = forward(layer, x, cu, positions)
        return backward(layer, y, saved)

    print(f"training step, 2 x 4096 tokens of width 4096, 32 heads of 128 sharing 8: {seconds(step) * 1e3:.2f} ms", flush=True)
    server, one = Server(layer, 32, 8192), x[:32].contiguous()
    server.lengths += 4000                                 # as if so many were there
    print(f"a token for 32 sequences of 4000 (their cache empty pages): {seconds(lambda: server.token(one)) * 1e6:.0f} us", flush=True)


if __name__ == "__main__":
    main()
