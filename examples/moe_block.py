"""A transformer's mixture-of-experts block from the residual stream to the residual
stream, served for a few tokens and trained.

    python examples/moe_block.py [--tokens 256] [--steps 10]

Serving: blocks of norm, router, experts and residual join decode up to 16 tokens,
with their weights in bf16 and in 4 bits (block.layer_few), eagerly and as one
replayed graph; prints what a block takes.  Training: the same blocks with norms on both
sides, a learnt gate for each channel and dropout, through the library's kernels and
their gradients; prints the loss.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_07536_amd import autograd, binding, block, experts  # noqa: E402


class ServedBlock:
    """One block's weights, as they are kept for serving."""

    def __init__(self, H, I, E, topk, gen, four_bits):
        def normal(*shape, scale=1.0):
            return torch.randn(shape, device="cuda", generator=gen) * scale
        self.topk = topk
        self.before = 1 + normal(H, scale=0.1)
        self.router = normal(H, E, scale=H ** -0.5).bfloat16()
        w1, w2 = normal(E, H, 2 * I, scale=H ** -0.5).bfloat16(), normal(E, I, H, scale=I ** -0.5).bfloat16()
        self.w_gate_up, self.w2 = w1, w2
        if four_bits:
            self.weights = experts.mx4_quantize_weights(w1), experts.mx4_quantize_weights(w2)
        else:
            self.weights = binding.pack_w1(w1), w2


def decode(blocks, h, scale=0.25):
    """h bf16 [T, H], T up to 16, through the blocks: the stream after the last one."""
    y = None
    for b in blocks:
        h, x = block.join(h, y, scale=scale, before=b.before)
        choice = block.choose((x @ b.router).float(), b.topk)
        y = block.layer_few(x, *b.weights, *choice)
    return block.join(h, y, scale=scale).h


def microseconds(call, n=50):
    for _ in range(5):
        call()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(n):
        call()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) * 1e3 / n


def serve(T=1, H=2048, I=704, E=32, topk=6, n=4, four_bits=False):
    gen = torch.Generator(device="cuda").manual_seed(0)
    blocks = [ServedBlock(H, I, E, topk, gen, four_bits) for _ in range(n)]
    h = torch.randn(T, H, device="cuda", generator=gen).bfloat16()
    want = decode(blocks, h)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        decode(blocks, h)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = decode(blocks, h)
    graph.replay()
    same = torch.equal(out, want)
    print(f"serving {T} tokens, weights in {'4 bits' if four_bits else 'bf16'}: a block eagerly "
          f"{microseconds(lambda: decode(blocks, h)) / n:.1f} us, replayed {microseconds(graph.replay) / n:.1f} us", flush=True)
    return same, want, blocks, h


class Block(torch.nn.Module):
    """Norm, router, SwiGLU experts, norm, gate, dropout and residual; fp32 master weights."""

    def __init__(self, H, I, E, topk, drop):
        super().__init__()
        self.topk, self.E, self.drop = topk, E, drop
        self.before = torch.nn.Parameter(torch.ones(H))
        self.after = torch.nn.Parameter(torch.ones(H))
        self.gate = torch.nn.Parameter(torch.full((1, H), 0.5))
        self.router = torch.nn.Parameter(torch.randn(H, E) * H ** -0.5)
        self.w1 = torch.nn.Parameter(torch.randn(E, H, 2 * I) * H ** -0.5)
        self.w2 = torch.nn.Parameter(torch.randn(E, I, H) * I ** -0.5)

    def forward(self, h, rng):
        h, x = autograd.join(h, before=self.before)
        ids, gates = autograd.choose(x.float() @ self.router, self.topk)
        r = experts.sort_by_expert(ids, gates.detach(), self.E)
        rows = autograd.dispatch(x, r)
        ys = []
        for e, row in enumerate(rows.split(r.expert_offsets.diff().tolist())):
            g, u = (row @ self.w1[e].bfloat16()).float().chunk(2, -1)
            ys.append((torch.nn.functional.silu(g) * u).bfloat16() @ self.w2[e].bfloat16())
        y = autograd.combine(torch.cat(ys), r, gates)
        return autograd.join(h, y, after=self.after, gate=self.gate, drop=self.drop if self.training else 0.0, rng=rng).h


def train(T, steps, H=256, I=128, E=8, topk=2, n=2, drop=0.1):
    torch.manual_seed(0)
    blocks = torch.nn.ModuleList([Block(H, I, E, topk, drop) for _ in range(n)]).cuda()
    other = torch.nn.ModuleList([Block(H, I, E, topk, 0.0) for _ in range(n)]).cuda().eval()
    opt = torch.optim.Adam(blocks.parameters(), lr=2e-3)
    losses = []
    for step in range(steps):
        # dropout's numbers: a seed for each block, an offset for each step
        rngs = torch.tensor([[17 + i, step] for i in range(n)], device="cuda")
        h = torch.randn(T, H, device="cuda").bfloat16()
        with torch.no_grad():
            want = h
            for b in other:
                want = b(want, None)
        out = h
        for b, rng in zip(blocks, rngs):
            out = b(out, rng)
        loss = (out.float() - want.float()).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
        print(f"training step {step}: loss {losses[-1]:.4f}", flush=True)
    return losses, blocks


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=256)
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args()
    for T in (1, 16):
        serve(T)
        serve(T, four_bits=True)
    train(a.tokens, a.steps)
