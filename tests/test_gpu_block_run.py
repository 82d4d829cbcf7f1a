"""GPU: the operators around and inside a block run together as a program runs them -
eagerly, on a stream of its own, replayed from a graph -, their differentiable forms, and
the example."""
import os
import sys

import numpy as np
import pytest

from oracle import block as ob

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


def _f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("T", [1, 5, 16])
@pytest.mark.parametrize("four_bits", [False, True])
def test_blocks_served_eagerly_and_from_a_graph(gpu_lib, T, four_bits):
    """The replay gives the eager bits, and the blocks, one by one on the inputs that
    they had, the oracle's (block.layer_few and block.join are tested to their bounds
    elsewhere; here the chain is what matters)."""
    import moe_block
    import torch

    from paper_2609_07536_amd import block as K
    from paper_2609_07536_amd import experts as X
    same, want, blocks, h = moe_block.serve(T, H=256, I=64, E=8, topk=2, n=3, four_bits=four_bits)
    assert same
    y = None
    for b in blocks:
        x, z = K.join(h, y, scale=0.25, before=b.before)
        if y is not None:
            exact = ob.join(_f64(h), _f64(y), None, None, 0.25)[0]
            assert (np.abs(_f64(x) - exact) <= 2.0 ** -8 * (np.abs(exact) + 1e-3)).all()
        logits = (z @ b.router).float()
        c = K.choose(logits, 2)
        ids, gates = ob.choose(_f64(logits), 2)
        assert np.array_equal(c.expert_ids.cpu().numpy(), ids) and np.abs(_f64(c.gates) - gates).max() < 1e-5
        y = K.layer_few(z, *b.weights, *c)
        if four_bits:
            w1, w2 = (_f64(X.mx4_dequantize(w, dtype=torch.float32)).transpose(0, 2, 1) for w in b.weights)
        else:
            w1, w2 = _f64(b.w_gate_up), _f64(b.w2)
        exact, tol = ob.layer(_f64(z), w1, w2, ids, _f64(c.gates))
        assert (np.abs(_f64(y) - exact) <= tol + 2.0 ** -24 * np.abs(exact)).all()
        h = x
    assert torch.equal(K.join(h, y, scale=0.25).h, want)


def test_replays_with_eager_work_between(gpu_lib):
    """Each replay, with other inputs and the program's own work and waits between, is the
    eager result; two graphs with scratch of their own."""
    import torch

    from paper_2609_07536_amd import binding as B
    from paper_2609_07536_amd import block as K
    gen = torch.Generator(device="cuda").manual_seed(1)
    H, I, E, k = 256, 64, 16, 4
    w1 = B.pack_w1(torch.randn(E, H, 2 * I, device="cuda", generator=gen).mul(H ** -0.5).bfloat16())
    w2 = torch.randn(E, I, H, device="cuda", generator=gen).mul(I ** -0.5).bfloat16()
    w = torch.rand(H, device="cuda", generator=gen)
    rng = torch.tensor([3, 0], device="cuda")
    graphs = []
    for T in (3, 16):
        h, l = torch.zeros(T, H, device="cuda"), torch.zeros(T, E, device="cuda")
        d = torch.zeros(T, H, device="cuda")
        scratch = torch.empty(K.layer_few_scratch_size(T, H, I, E, k), dtype=torch.uint8, device="cuda")
        sums = torch.empty(K.join_grad_scratch_size(T, H), dtype=torch.uint8, device="cuda")

        def run(h=h, l=l, d=d, scratch=scratch, sums=sums):
            c = K.choose(l, k, score="sigmoid")
            y = K.layer_few(K.join(h, before=w).z, w1, w2, *c, scratch=scratch)
            x, z = K.join(h, y, after=w, drop=0.25, rng=rng, before=w, dtype=torch.float32)
            g = K.join_grad(d, z, x, y, after=w, drop=0.25, rng=rng, before=w, scratch=sums)
            return [*c, y, x, z, *(t for t in g if t is not None), K.choose_grad(c.gates, l, c.expert_ids, score="sigmoid")]
        run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run()
        graphs.append((g, (h, l, d), run, out))
    for i in range(6):
        for g, inputs, run, out in graphs:
            for t in inputs:
                t.normal_(generator=gen)
            rng[1] = i
            g.replay()
            eager = run()
            torch.cuda.synchronize()
            for a, b in zip(out, eager):
                assert torch.equal(a, b)


def test_on_a_stream_of_its_own(gpu_lib):
    """Work on a given stream waits for what that stream waits for, and for nothing else."""
    import torch

    from paper_2609_07536_amd import binding as B
    from paper_2609_07536_amd import block as K
    gen = torch.Generator(device="cuda").manual_seed(2)
    H, I, E, k, T = 512, 96, 8, 2, 9
    w1 = B.pack_w1(torch.randn(E, H, 2 * I, device="cuda", generator=gen).mul(H ** -0.5).bfloat16())
    w2 = torch.randn(E, I, H, device="cuda", generator=gen).mul(I ** -0.5).bfloat16()
    w = torch.rand(H, device="cuda", generator=gen)
    h, l = torch.randn(T, H, device="cuda", generator=gen), torch.randn(T, E, device="cuda", generator=gen)
    s = torch.cuda.Stream()

    def run(stream):
        c = K.choose(l, k, stream=stream)
        z = K.join(h, before=w, stream=stream).z
        y = K.layer_few(z, w1, w2, *c, stream=stream)
        x, z = K.join(h, y, before=w, stream=stream)
        g = K.join_grad(x, z, x, y, before=w, stream=stream)
        return [*c, y, x, z, g.h, g.y, g.before, K.choose_grad(c.gates, l, c.expert_ids, stream=stream)]
    want = run(None)
    for _ in range(5):
        s.wait_stream(torch.cuda.current_stream())
        got = run(s)
        s.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_differentiable_choose(gpu_lib):
    """Against torch's own operations in 64 bits, gradients among them."""
    import torch

    from paper_2609_07536_amd import autograd as A
    gen = torch.Generator(device="cuda").manual_seed(3)
    l = torch.randn(70, 20, device="cuda", generator=gen)
    d = torch.randn(70, 4, device="cuda", generator=gen)
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            a, b = l.clone().requires_grad_(), l.double().requires_grad_()
            ids, gates = A.choose(a, 4, score=score, renormalize=renorm, scale=1.5)
            assert not ids.requires_grad
            (gates * d).sum().backward()
            p = torch.softmax(b, -1) if score == "softmax" else torch.sigmoid(b)
            q = p.gather(1, ids.long())
            q = 1.5 * (q / q.sum(1, keepdim=True) if renorm else q)
            (q * d.double()).sum().backward()
            # (scores of logits within 10 of each other, sums of 20 terms: the bounds of test_gpu_block.py)
            assert torch.allclose(gates.double(), q, rtol=60 * 2.0 ** -24, atol=0)
            assert (a.grad.double() - b.grad).abs().max() <= 200 * 2.0 ** -24 * d.abs().max() * 4
    ids, gates = A.choose(l.clone().requires_grad_(), 4)
    (ids.sum() + gates.detach().sum()).item()     # (nothing to differentiate, no error)


@pytest.mark.parametrize("kind", ["none", "token", "channel"])
@pytest.mark.parametrize("after,before", [(True, True), (False, True), (True, False), (False, False)])
def test_differentiable_join(gpu_lib, kind, after, before):
    """Against torch's own operations in 64 bits; in fp32, whose errors here (sums of up to
    130 terms of size 1 to 10, weights near 1) are far below 1e-4 of the gradients' scale."""
    import torch

    from paper_2609_07536_amd import autograd as A
    gen = torch.Generator(device="cuda").manual_seed(4)

    def leaf(*shape):
        return torch.randn(shape, device="cuda", generator=gen)
    T, H, p = 50, 130, 0.25
    leaves = dict(h=leaf(T, H), y=leaf(T, H), after=1 + leaf(H) / 4 if after else None,
                  gate={"none": None, "token": leaf(T, 1), "channel": leaf(1, H)}[kind],
                  before=1 + leaf(H) / 4 if before else None)
    rng = torch.tensor([5, 6], device="cuda")
    mask = torch.from_numpy(ob.kept(5, 6, T, H, p)).cuda()
    a = {k: None if v is None else v.clone().requires_grad_() for k, v in leaves.items()}
    b = {k: None if v is None else v.double().requires_grad_() for k, v in leaves.items()}
    x, z = A.join(a["h"], a["y"], a["after"], a["gate"], 0.7, p, rng, a["before"], dtype=torch.float32)
    rng += 1     # (the next call's numbers: this one's are kept)
    c = b["y"]
    if after:
        c = c * torch.rsqrt(c.square().mean(1, keepdim=True) + 1e-6) * b["after"]
    c = c if b["gate"] is None else c * b["gate"]
    wx = b["h"] + 0.7 * mask * c
    wz = wx * torch.rsqrt(wx.square().mean(1, keepdim=True) + 1e-6) * b["before"] if before else None
    dx, dz = leaf(T, H), leaf(T, H)
    ((x * dx).sum() + ((z * dz).sum() if before else 0.0)).backward()
    ((wx * dx.double()).sum() + ((wz * dz.double()).sum() if before else 0.0)).backward()
    assert (z is None) == (not before)
    for k in a:
        if a[k] is not None:
            assert a[k].grad.dtype == a[k].dtype
            off = (a[k].grad.double() - b[k].grad).abs().max() / b[k].grad.abs().max()
            assert off <= 1e-4, (k, float(off))


def test_differentiable_join_of_what_is_not_asked_for(gpu_lib):
    """Only some gradients, only the norm's output used, the norm alone, h None, bf16
    weights, strided inputs."""
    import torch

    from paper_2609_07536_amd import autograd as A
    h, y = torch.randn(9, 40, device="cuda"), torch.randn(40, 9, device="cuda").t()
    w = torch.rand(40, device="cuda").bfloat16().requires_grad_()
    hh = h.clone().requires_grad_()
    z = A.join(hh, y, after=w, before=w).z
    z.float().sum().backward()
    assert w.grad.dtype == torch.bfloat16 and hh.grad.shape == h.shape
    out = A.join(hh, before=w)
    assert out.h is hh
    (out.h.sum() + out.z.float().sum()).backward()
    yy = torch.randn(9, 40, device="cuda", requires_grad=True)
    rng = torch.tensor([1, 2], device="cuda")
    r = A.join(None, yy, drop=0.5, rng=rng).h
    r.sum().backward()
    assert torch.equal((yy.grad != 0), (r != 0)) and torch.equal(yy.grad[yy.grad != 0].unique(), torch.tensor([2.0], device="cuda"))
    x, z = A.join(hh.detach(), yy, before=w)
    (x.sum() * 0 + 1).backward()
    assert not bool((yy.grad[r == 0] != 0).any())


def test_a_saved_stream_that_a_call_wrote_to_is_refused(gpu_lib):
    """As after torch's own in-place operations: an error, not another gradient."""
    import torch

    from paper_2609_07536_amd import autograd as A
    from paper_2609_07536_amd import block as K
    h, y, w = torch.randn(4, 64, device="cuda"), torch.randn(4, 64, device="cuda"), torch.rand(64, device="cuda")
    x, z = A.join(h.requires_grad_(), y, before=w)
    with torch.no_grad():
        K.join(x, y, out=K.Joined(x, None))
    with pytest.raises(RuntimeError, match="inplace"):
        z.float().sum().backward()
    l = torch.randn(4, 8, device="cuda", requires_grad=True)
    ids, gates = A.choose(l, 2)
    with torch.no_grad():
        K.choose(l.detach(), 2, out=K.Choice(ids, gates.detach()))
    with pytest.raises(RuntimeError, match="inplace"):
        gates.sum().backward()


def test_every_given_output_counts_as_changed(gpu_lib):
    import torch

    from paper_2609_07536_amd import binding as B
    from paper_2609_07536_amd import block as K
    T, H, I, E, k = 4, 64, 32, 4, 2
    h, y, l, w = (torch.randn(s, device="cuda") for s in ((T, H), (T, H), (T, E), (H,)))
    ids, g = K.choose(l, k)
    w1, w2 = B.pack_w1(torch.randn(E, H, 2 * I, device="cuda").bfloat16()), torch.randn(E, I, H, device="cuda").bfloat16()
    x = h.bfloat16()
    calls = [(lambda o: K.choose(l, k, out=K.Choice(*o)), [ids.clone(), g.clone()]),
             (lambda o: K.choose_grad(g, l, ids, out=o[0]), [l.clone()]),
             (lambda o: K.join(h, y, before=w, out=K.Joined(*o)), [h.clone(), x.clone()]),
             (lambda o: K.join_grad(h, h, h, y, after=w, gate=w[None], before=w, out=K.JoinGrads(*o)),
              [h.clone(), y.clone(), w.clone(), w[None].clone(), w.clone()]),
             (lambda o: K.layer_few(x, w1, w2, ids, g, out=o[0]), [h.clone()])]
    inputs = [h, y, l, w, ids, g, w1, w2, x]
    for call, outs in calls:
        before = [t._version for t in inputs]
        v = [t._version for t in outs]
        call(outs)
        assert all(t._version > n for t, n in zip(outs, v)) and [t._version for t in inputs] == before


def test_training_step_captured_and_replayed(gpu_lib):
    """A forward and backward pass of differentiable choose and join in one graph, its
    gradients those of the eager pass."""
    import torch

    from paper_2609_07536_amd import autograd as A
    T, H, E = 64, 96, 8
    h, y, l = (torch.randn(s, device="cuda").requires_grad_() for s in ((T, H), (T, H), (T, E)))
    w = torch.rand(H, device="cuda").requires_grad_()
    rng = torch.tensor([7, 0], device="cuda")

    def step():
        x, z = A.join(h, y, after=w, drop=0.2, rng=rng, before=w)
        ids, gates = A.choose(l, 2)
        loss = x.square().sum() + z.float().sum() + gates.square().sum()
        return torch.autograd.grad(loss, (h, y, l, w))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(4):
        with torch.no_grad():
            h.normal_(), y.normal_(), l.normal_()
        rng[1] = i
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b)


def test_example(gpu_lib):
    import moe_block
    import torch
    losses, blocks = moe_block.train(96, 3, H=64, I=32, E=4, topk=2)
    assert len(losses) == 3 and all(np.isfinite(losses))
    for name, p in blocks.named_parameters():
        assert p.grad is not None and bool(torch.isfinite(p.grad).all()) and float(p.grad.abs().max()) > 0, name


def test_differentiable_join_refuses_dropout_without_numbers(gpu_lib):
    import torch

    from paper_2609_07536_amd import autograd as A
    x = torch.zeros(4, 8, device="cuda")
    with pytest.raises(TypeError, match="rng: dropout needs one"):
        A.join(x, x, drop=0.5)


@pytest.mark.parametrize("used", ["z", "x", "both"])
@pytest.mark.parametrize("kind", ["norm alone", "none", "token", "channel"])
def test_differentiable_join_by_what_is_used(gpu_lib, used, kind):
    """Every leaf's gradient where the stream alone, its norm alone, or both are used, of the
    join and of the norm alone, against torch's own operations in 64 bits: in fp32, within the
    1e-4 of test_differentiable_join's sizes.  A leaf that what is used does not depend on
    has zeros or no gradient."""
    import torch

    from paper_2609_07536_amd import autograd as A
    gen = torch.Generator(device="cuda").manual_seed(6)

    def leaf(*shape):
        return torch.randn(shape, device="cuda", generator=gen)
    T, H, with_y = 50, 130, kind != "norm alone"
    leaves = dict(h=leaf(T, H), y=leaf(T, H) if with_y else None, after=1 + leaf(H) / 4 if with_y else None,
                  gate={"token": leaf(T, 1), "channel": leaf(1, H)}.get(kind), before=1 + leaf(H) / 4)
    a = {k: None if v is None else v.clone().requires_grad_() for k, v in leaves.items()}
    b = {k: None if v is None else v.double().requires_grad_() for k, v in leaves.items()}
    x, z = A.join(a["h"], a["y"], a["after"], a["gate"], scale=0.7 if with_y else 1.0, before=a["before"], dtype=torch.float32)
    wx = b["h"]
    if with_y:
        c = b["y"] * torch.rsqrt(b["y"].square().mean(1, keepdim=True) + 1e-6) * b["after"]
        wx = wx + 0.7 * (c if b["gate"] is None else c * b["gate"])
    wz = wx * torch.rsqrt(wx.square().mean(1, keepdim=True) + 1e-6) * b["before"]
    dx, dz = leaf(T, H) * (used != "z"), leaf(T, H) * (used != "x")
    (((x * dx).sum() if used != "z" else 0.0) + ((z * dz).sum() if used != "x" else 0.0)).backward()
    ((wx * dx.double()).sum() + (wz * dz.double()).sum()).backward()
    for k in a:
        if a[k] is None:
            continue
        want = b[k].grad
        if not bool(want.any()):
            assert used == "x" and k == "before" and (a[k].grad is None or not bool(a[k].grad.any()))
            continue
        off = (a[k].grad.double() - want).abs().max() / want.abs().max()
        assert off <= 1e-4, (k, float(off))


@pytest.mark.parametrize("y_type", ["bfloat16", "float32"])
def test_backward_of_a_join_takes_no_memory_beside_its_gradients(gpu_lib, y_type):
    """y is not read again without a norm after the block and a gate: the backward pass has
    room for the gradients of h and y and, but for 1 MiB, for nothing else."""
    import torch

    from paper_2609_07536_amd import autograd as A
    T, H = 4096, 1024
    h = torch.randn(T, H, device="cuda").requires_grad_()
    y = torch.randn(T, H, device="cuda").to(getattr(torch, y_type)).requires_grad_()
    x, z = A.join(h, y, scale=0.5, before=torch.ones(H, device="cuda"))
    dx, dz = torch.randn_like(x), torch.randn_like(z)
    want = h.numel() * h.element_size() + y.numel() * y.element_size()
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    base = torch.cuda.memory_allocated()
    gh, gy = torch.autograd.grad((x, z), (h, y), (dx, dz))
    assert torch.cuda.max_memory_allocated() - base <= want + 2 ** 20
    assert torch.equal(gy, (0.5 * gh).to(y.dtype))
    # a block's output without a gradient, dropout and all
    rng = torch.tensor([1, 2], device="cuda")
    x, z = A.join(h, y.detach(), scale=0.5, drop=0.25, rng=rng, before=torch.ones(H, device="cuda"))
    g, = torch.autograd.grad(x, h, dx)
    assert torch.equal(g, dx)
