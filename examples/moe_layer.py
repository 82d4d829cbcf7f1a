"""A mixture-of-experts layer from its router on, served and trained.

    python examples/moe_layer.py [--tokens 1024] [--steps 20]

Serving: the router's top-k is sorted by expert, and the layer runs with its
experts in bf16 (binding.layer_forward) and in 4 bits (experts.layer_forward_mx4);
prints how far the two are apart and what a call of each takes.  Training: a
layer with learnt router and experts fits another one, its tokens dispatched and
combined by the library's kernels with their gradients; prints the loss.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_07536_amd import autograd, binding, experts  # noqa: E402


def route(hidden, router, topk):
    """A softmax router's choice: expert ids and renormalised gates [T, topk]."""
    p, ids = torch.softmax(hidden.float() @ router, -1).topk(topk, -1)
    return ids.int(), p / p.sum(-1, keepdim=True)


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


def serve(T, H=2048, I=704, E=32, topk=6):
    gen = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, device="cuda", generator=gen) * scale
    hidden, router = normal(T, H).bfloat16(), normal(H, E, scale=H ** -0.5)
    w_gate_up, w2 = normal(E, H, 2 * I, scale=H ** -0.5).bfloat16(), normal(E, I, H, scale=I ** -0.5).bfloat16()
    # once, as the weights are loaded
    w1, w1_4, w2_4 = binding.pack_w1(w_gate_up), experts.mx4_quantize_weights(w_gate_up), experts.mx4_quantize_weights(w2)
    wl, _ = binding.make_workload(T, H, I, E, topk, 1, rows=T * topk)
    ws = binding.Workspace(binding.layer_workspace_size(wl))
    scratch = torch.empty(experts.mx4_layer_scratch_size(T, H, I, topk), dtype=torch.uint8, device="cuda")
    out16, out4 = torch.empty(T, H, device="cuda"), torch.empty(T, H, device="cuda")

    ids, gates = route(hidden, router, topk)
    r = experts.sort_by_expert(ids, gates, E)
    sort = lambda: experts.sort_by_expert(ids, gates, E, out=r)  # noqa: E731
    bf16 = lambda: binding.layer_forward(hidden, w1, w2, r.expert_offsets, r.token_ids, r.gate_w, topk,  # noqa: E731
                                         out=out16, workspace=ws)
    four = lambda: experts.layer_forward_mx4(hidden, w1_4, w2_4, r, gates, out=out4, scratch=scratch,  # noqa: E731
                                             workspace=ws)
    bf16(), four()
    assert ws.status() == 0
    off = float((out4 - out16).norm() / out16.norm())
    print(f"serving {T} tokens: sort {microseconds(sort):.1f} us, layer in bf16 {microseconds(bf16):.1f} us, in 4 bits "
          f"{microseconds(four):.1f} us, outputs {off:.3f} apart", flush=True)
    return off, out4, (hidden, w_gate_up, w2, ids, gates)


class Layer(torch.nn.Module):
    """SwiGLU experts in bf16 with fp32 master weights, a softmax router."""

    def __init__(self, H, I, E, topk):
        super().__init__()
        self.topk, self.E = topk, E
        self.router = torch.nn.Parameter(torch.randn(H, E) * H ** -0.5)
        self.w1 = torch.nn.Parameter(torch.randn(E, H, 2 * I) * H ** -0.5)
        self.w2 = torch.nn.Parameter(torch.randn(E, I, H) * I ** -0.5)

    def forward(self, x):
        ids, gates = route(x, self.router, self.topk)
        r = experts.sort_by_expert(ids, gates.detach(), self.E)
        rows = autograd.dispatch(x, r)
        ys = []
        for e, row in enumerate(rows.split(r.expert_offsets.diff().tolist())):
            g, u = (row @ self.w1[e].bfloat16()).float().chunk(2, -1)
            ys.append((torch.nn.functional.silu(g) * u).bfloat16() @ self.w2[e].bfloat16())
        return autograd.combine(torch.cat(ys), r, gates)


def train(T, steps, H=256, I=128, E=8, topk=2):
    torch.manual_seed(0)
    layer, other = Layer(H, I, E, topk).cuda(), Layer(H, I, E, topk).cuda()
    opt = torch.optim.Adam(layer.parameters(), lr=2e-3)
    losses = []
    for step in range(steps):
        x = torch.randn(T, H, device="cuda").bfloat16()
        with torch.no_grad():
            want = other(x)
        loss = (layer(x) - want).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
        print(f"training step {step}: loss {losses[-1]:.4f}", flush=True)
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    serve(a.tokens)
    train(a.tokens, a.steps)
