"""GPU: the sort by expert, the rows' way to the experts and back, and its
gradients, against the 64-bit oracle and (gradients) against differences.

Tolerances.  fp32 sums of n terms in any order are off by at most
n 2^-24 times the sum of the terms' magnitudes; rounding to bf16 adds 2^-8 of
the value (a half unit is 2^-9), to fp32 2^-24.
"""
import numpy as np
import pytest

from oracle import experts as oe

pytestmark = pytest.mark.gpu
ROUND = {"bfloat16": 2.0 ** -8, "float32": 2.0 ** -23}


def _X():
    from paper_2609_07536_amd import experts
    return experts


def _choice(rng, T, k, E, drop=0.0, repeat=False):
    if repeat:
        ids = rng.integers(0, E, (T, k))
    else:
        ids = np.argsort(rng.random((T, E)), 1)[:, :k]
    ids = ids.astype(np.int32)
    lost = rng.random((T, k)) < drop
    ids[lost] = rng.choice([-1, E, -2 ** 31, 2 ** 31 - 1], int(lost.sum()))
    return ids, rng.random((T, k), dtype=np.float32)


def _cuda(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(getattr(torch, dtype))


def _shifted(t, by):
    """The same values in memory that starts `by` elements after an aligned address."""
    import torch
    base = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")
    v = base[by:].view(t.shape)
    v.copy_(t)
    return v


def _f64(t):
    return t.double().cpu().numpy()


def _rows_case(seed, T, k, H, E=8, drop=0.2, extra=0):
    """ids, slot_rows and a number of rows with `extra` rows that no slot has."""
    rng = np.random.default_rng(seed)
    ids, gates = _choice(rng, T, k, max(E, k), drop)
    rows = oe.sort_by_expert(ids, gates, max(E, k))[3]
    gates = gates * rng.choice([-1.0, 1.0], gates.shape).astype(np.float32)
    return rng, rows, gates, int((rows >= 0).sum()) + extra


@pytest.mark.parametrize("T,k,E,drop", [
    (1, 1, 1, 0.0), (1, 6, 32, 0.0), (1, 6, 32, 1.0), (7, 3, 11, 0.3), (64, 6, 32, 0.0), (65, 1, 2, 0.1),
    (512, 8, 1024, 0.1), (4096, 1, 513, 0.0), (682, 6, 32, 0.0), (683, 6, 32, 0.2), (4097, 1, 1, 0.0),
    (777, 64, 100, 0.2), (2048, 8, 1024, 0.05), (5003, 5, 300, 0.9), (16384, 6, 32, 0.05)])
def test_sort(gpu_lib, T, k, E, drop):
    import torch
    X = _X()
    ids, gates = _choice(np.random.default_rng([T, k, E]), T, k, E, drop)
    want = oe.sort_by_expert(ids, gates, E)
    out = X.Routing(*(torch.full(s, 77, dtype=d, device="cuda") for s, d in (
        ((E + 1,), torch.int32), ((T * k,), torch.int32), ((T * k,), torch.float32), ((T, k), torch.int32))))
    got = X.sort_by_expert(_cuda(ids), _cuda(gates), E, out=out)
    for name, g, w in zip(X.Routing._fields, got, want):
        assert np.array_equal(g.cpu().numpy(), w), name


@pytest.mark.parametrize("first,E", [(0, 8), (8, 8), (56, 8), (-3, 5), (2 ** 31 - 4, 8)])
@pytest.mark.parametrize("T", [40, 3000])
def test_sort_of_a_share_of_the_experts(gpu_lib, T, first, E):
    """Expert parallelism: the ids of another GPU's experts are slots without a
    row; a token may name an expert twice."""
    X = _X()
    rng = np.random.default_rng(T)
    ids, gates = _choice(rng, T, 4, 64, 0.1, repeat=True)
    ids[::3] = np.minimum(np.int64(first) + rng.integers(0, E, ids[::3].shape), 2 ** 31 - 1)
    got = X.sort_by_expert(_cuda(ids), _cuda(gates), E, first_expert=first)
    for g, w in zip(got, oe.sort_by_expert(ids, gates, E, first)):
        assert np.array_equal(g.cpu().numpy(), w)


def test_sort_of_one_hot_expert(gpu_lib):
    X = _X()
    ids = np.full((30000, 2), 5, np.int32)
    gates = np.random.default_rng(0).random(ids.shape, dtype=np.float32)
    got = X.sort_by_expert(_cuda(ids), _cuda(gates), 7)
    assert got.expert_offsets.tolist() == [0] * 6 + [60000] * 2
    assert np.array_equal(got.slot_rows.cpu().numpy().ravel(), np.arange(60000))
    assert np.array_equal(got.gate_w.cpu().numpy(), gates.ravel())


def test_sort_of_more_slots_than_chunks_of_the_usual_size(gpu_lib):
    """2.4 million slots: chunks grow so that their number stays bounded."""
    import torch
    X = _X()
    ids = torch.randint(-1, 40, (300000, 8), dtype=torch.int32, device="cuda")
    gates = torch.rand(300000, 8, device="cuda")
    r = X.sort_by_expert(ids, gates, 40)
    flat = ids.view(-1).cpu().numpy()
    order = np.argsort(np.where(flat < 0, 40, flat), kind="stable")[:int((flat >= 0).sum())]
    assert np.array_equal(r.token_ids.cpu().numpy()[:len(order)], order // 8)
    assert bool((r.token_ids[len(order):] == -1).all()) and bool((r.gate_w[len(order):] == 0).all())
    assert np.array_equal(r.slot_rows.view(-1).cpu().numpy()[order], np.arange(len(order)))
    assert np.array_equal(r.expert_offsets.cpu().numpy()[1:], np.cumsum(np.bincount(flat[flat >= 0], minlength=40)))


def test_no_tokens(gpu_lib):
    import torch
    X = _X()
    e = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    g = torch.empty((0, 4), device="cuda")
    r = X.sort_by_expert(e, g, 5)
    assert r.expert_offsets.tolist() == [0] * 6 and r.token_ids.numel() == 0
    x = torch.empty((0, 16), device="cuda")
    assert X.dispatch_rows(x, e, 0).shape == (0, 16)
    assert X.combine_rows(x, e, g).shape == (0, 16)
    assert [t.shape[0] for t in X.combine_rows_grad(x, x, e, g)] == [0, 0]
    # tokens, but no rows: sums of nothing
    none = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    assert X.combine_rows(x, none, torch.ones(3, 4, device="cuda")).tolist() == [[0.0] * 16] * 3
    assert X.dispatch_rows_grad(x, none).tolist() == [[0.0] * 16] * 3
    assert X.combine_rows_grad(torch.ones(3, 16, device="cuda"), x, none, torch.ones(3, 4, device="cuda"))[1].tolist() == [[0.0] * 4] * 3


@pytest.mark.parametrize("T,k,H", [(1, 6, 2048), (5, 1, 1), (9, 3, 7), (33, 8, 8), (65, 2, 9), (30, 64, 130),
                                   (777, 3, 1352), (17, 5, 511), (70, 4, 2049), (20, 6, 4100)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32", "uint8"])
@pytest.mark.parametrize("by", [0, 3])
def test_dispatch(gpu_lib, T, k, H, dtype, by):
    import torch
    X = _X()
    rng, rows, _, M = _rows_case([T, k, H], T, k, H, extra=2)
    x = rng.integers(0, 200, (T, H)).astype(np.float64)
    dx = _shifted(_cuda(x, dtype), by)
    out = _shifted(torch.full((M, H), 99, dtype=dx.dtype, device="cuda"), by)
    got = X.dispatch_rows(dx, _cuda(rows), M, out=out)
    assert np.array_equal(_f64(got), oe.dispatch(x, rows, np.full((M, H), 99.0)))


SHAPES = [(1, 6, 2048), (5, 1, 1), (9, 3, 7), (33, 8, 8), (65, 2, 9), (12, 64, 130), (300, 3, 1352),
          (17, 5, 511), (40, 4, 2049), (20, 9, 4100)]


@pytest.mark.parametrize("T,k,H", SHAPES)
@pytest.mark.parametrize("src,dst", [("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float32", "bfloat16"),
                                     ("float32", "float32")])
@pytest.mark.parametrize("by", [0, 1])
def test_combine_and_dispatch_grad(gpu_lib, T, k, H, src, dst, by):
    import torch
    X = _X()
    rng, rows, gates, M = _rows_case([T, k, H], T, k, H, extra=1)
    y = _shifted(_cuda(rng.standard_normal((M, H)), src), by)
    y[M - 1] = float("nan")      # the row that no slot has
    for weighted in (True, False):
        out = _shifted(torch.full((T, H), float("nan"), dtype=getattr(torch, dst), device="cuda"), by)
        if weighted:
            got = X.combine_rows(y, _cuda(rows), _cuda(gates), out=out)
        else:
            got = X.dispatch_rows_grad(y, _cuda(rows), out=out)
        want, mag = oe.combine(_f64(y), rows, gates if weighted else None)
        assert (np.abs(_f64(got) - want) <= 2 * k * 2.0 ** -24 * mag + ROUND[dst] * np.abs(want)).all()


@pytest.mark.parametrize("T,k,H", SHAPES)
@pytest.mark.parametrize("d,t", [("bfloat16", "bfloat16"), ("float32", "bfloat16"), ("bfloat16", "float32"),
                                 ("float32", "float32")])
@pytest.mark.parametrize("by", [0, 1])
def test_combine_grad(gpu_lib, T, k, H, d, t, by):
    import torch
    X = _X()
    rng, rows, gates, M = _rows_case([T, k, H], T, k, H, extra=1)
    y = _shifted(_cuda(rng.standard_normal((M, H)), t), by)
    do = _shifted(_cuda(rng.standard_normal((T, H)), d), by)
    out = (_shifted(torch.full((M, H), 7.0, dtype=y.dtype, device="cuda"), by),
           torch.full((T, k), float("nan"), device="cuda"))
    dy, dg = X.combine_rows_grad(do, y, _cuda(rows), _cuda(gates), out=out)
    want, wg, mag = oe.combine_grad(_f64(do), _f64(y), rows, gates)
    want[M - 1] = 7.0            # no slot has it: not written
    assert (np.abs(_f64(dy) - want) <= ROUND[t] * np.abs(want)).all()
    assert (np.abs(_f64(dg) - wg) <= H * 2.0 ** -24 * mag).all()
    assert (_f64(dg)[rows < 0] == 0).all()


def test_gradients_against_differences(gpu_lib):
    """combine is linear in y and in the gates and dispatch in x, so a central
    difference with step 1 is the derivative up to the forward pass's rounding
    (fp32 throughout here): k + 1 roundings of the sum of magnitudes."""
    X = _X()
    T, k, H = 37, 5, 333
    rng, rows, gates, M = _rows_case(9, T, k, H)
    y, vy, do, x, vx = (rng.standard_normal(s).astype(np.float32) for s in ((M, H), (M, H), (T, H), (T, H), (T, H)))
    vg = rng.standard_normal((T, k)).astype(np.float32)
    r, D = _cuda(rows), np.float64

    def loss(y, g):
        return float((_f64(X.combine_rows(_cuda(y), r, _cuda(g))) * do).sum())

    dy, dg = X.combine_rows_grad(_cuda(do), _cuda(y), r, _cuda(gates))
    for a, b, got in ((loss(y + vy, gates), loss(y - vy, gates), (_f64(dy) * vy).sum()),
                      (loss(y, gates + vg), loss(y, gates - vg), (_f64(dg) * vg).sum())):
        mag = (oe.combine(np.abs(y) + np.abs(vy), rows, np.abs(gates) + np.abs(vg))[0] * np.abs(do)).sum()
        assert abs((a - b) / 2 - got) <= 2 * (k + 3) * 2.0 ** -24 * mag
    d = rng.standard_normal((M, H)).astype(np.float32)
    dx = X.dispatch_rows_grad(_cuda(d), r)

    def through(x):
        return float((_f64(X.dispatch_rows(_cuda(x), r, M)) * d.astype(D)).sum())
    mag = (oe.combine(np.abs(d), rows)[0] * (np.abs(x) + np.abs(vx))).sum()
    assert abs((through(x + vx) - through(x - vx)) / 2 - (_f64(dx) * vx).sum()) <= 2 * (k + 3) * 2.0 ** -24 * mag


def test_rows_without_a_slot_and_slots_without_a_row_add_nothing(gpu_lib):
    """An infinity or NaN reaches exactly the tokens whose slots have its row."""
    import torch
    X = _X()
    rows = _cuda(np.array([[0, -1], [-1, -1], [2, 3]], np.int32))
    y = torch.ones(5, 600, device="cuda")
    y[1], y[4], y[3] = float("nan"), float("inf"), float("inf")
    gates = torch.tensor([[2.0, float("nan")], [float("inf"), float("nan")], [1.0, 1.0]], device="cuda")
    out = X.combine_rows(y, rows, gates)
    assert bool((out[0] == 2).all()) and bool((out[1] == 0).all()) and bool((out[2] == float("inf")).all())
    dy, dg = X.combine_rows_grad(torch.ones(3, 600, device="cuda"), y, rows, gates)
    assert dg.tolist() == [[600.0, 0.0], [0.0, 0.0], [600.0, float("inf")]]
    assert bool((dy[0] == 2).all())
    # an infinity in the columns that two chunks of a ragged row share, against zero
    y = torch.zeros(1, 603, device="cuda")
    y[0, 598] = float("inf")
    do = torch.ones(1, 603, device="cuda")
    one = _cuda(np.zeros((1, 1), np.int32))
    assert X.combine_rows_grad(do, y, one, torch.ones(1, 1, device="cuda"))[1].item() == float("inf")


def test_bad_rows_are_skipped_and_flagged(gpu_lib):
    import torch

    from paper_2609_07536_amd import binding as B
    X = _X()
    ws = B.Workspace(512)
    rows = _cuda(np.array([[0, 1], [2, 7], [-9, 3]], np.int32))
    gates, x = torch.ones(3, 2, device="cuda"), torch.arange(3, device="cuda").float()[:, None].expand(3, 40).contiguous()
    y = torch.ones(4, 40, device="cuda")
    good = _cuda(np.array([[0, 1], [2, -1], [-1, 3]], np.int32))
    calls = [lambda r: X.dispatch_rows(x, r, 4, workspace=ws), lambda r: X.combine_rows(y, r, gates, workspace=ws),
             lambda r: X.dispatch_rows_grad(y, r, workspace=ws),
             lambda r: X.combine_rows_grad(x, y, r, gates, workspace=ws)[1]]
    for call in calls:
        want = call(good)
        assert ws.status() == 0
        assert torch.equal(call(rows), want)
        assert ws.status(clear=True) == B.MOE_ERR_BAD_ROUTING


def test_rows_past_4_gib(gpu_lib):
    """Offsets past 32 bits: the last of 1.2 million rows of 2048 bf16 values."""
    import torch
    X = _X()
    M, H = 1_200_000, 2048
    rows = torch.tensor([[M - 1, 0], [M // 2, M - 2]], dtype=torch.int32, device="cuda")
    x = torch.randn(2, H, device="cuda").bfloat16()
    big = torch.zeros(M, H, dtype=torch.bfloat16, device="cuda")
    X.dispatch_rows(x, rows, M, out=big)
    for t in range(2):
        for r in rows[t].tolist():
            assert torch.equal(big[r], x[t])
    assert int((big[::3].abs().sum(1) > 0).sum()) == sum(r % 3 == 0 for r in rows.view(-1).tolist())
    g = torch.tensor([[2.0, 1.0], [1.0, 3.0]], device="cuda")
    assert torch.equal(X.combine_rows(big, rows, g), x.float() * g.sum(1, keepdim=True))
    dy, dg = X.combine_rows_grad(x, big, rows, g)
    assert torch.equal(dy[M - 1], (2 * x[0].float()).bfloat16())
    assert torch.allclose(dg, x.float().square().sum(1, keepdim=True).expand(2, 2), rtol=H * 2.0 ** -24)


def test_another_stream_and_a_graph(gpu_lib):
    """On a stream of the caller's, and captured: replays follow their inputs."""
    import torch
    X = _X()
    T, k, H, E = 900, 6, 264, 16
    rng = np.random.default_rng(3)
    ids, gates = (_cuda(a) for a in _choice(rng, T, k, E, 0.1))
    x = torch.randn(T, H, device="cuda").bfloat16()

    def all_of(stream=None, keep=None):
        r = X.sort_by_expert(ids, gates, E, stream=stream)
        rows = torch.empty((T * k, H), dtype=x.dtype, device="cuda") if keep is None else keep
        p = X.dispatch_rows(x, r.slot_rows, T * k, out=rows, stream=stream)
        out = X.combine_rows(p, r.slot_rows, gates, stream=stream)
        dy, dg = X.combine_rows_grad(out, p, r.slot_rows, gates, stream=stream)
        return [*r, out, dg, X.dispatch_rows_grad(p, r.slot_rows, stream=stream)]

    side = torch.cuda.Stream()
    keep = torch.empty((T * k, H), dtype=x.dtype, device="cuda")
    want = all_of()
    torch.cuda.synchronize()
    got = all_of(side, keep)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of(keep=keep)
    for seed in range(4):
        new, g = _choice(np.random.default_rng(seed), T, k, E, 0.1 * seed)
        ids.copy_(_cuda(new))
        gates.copy_(_cuda(g))
        x.copy_(torch.randn(T, H, device="cuda"))
        want = all_of()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


def test_the_layer_on_a_sorted_choice(gpu_lib):
    """layer_forward takes the sort's outputs as they are, with rows = T topk and
    fewer in use, and combine_rows gives what its combine gives."""
    import torch

    from paper_2609_07536_amd import binding as B
    X = _X()
    T, H, I, E, k = 200, 512, 64, 8, 3
    ids, gates = (_cuda(a) for a in _choice(np.random.default_rng(1), T, k, E, 0.2))
    r = X.sort_by_expert(ids, gates, E)
    gen = torch.Generator(device="cuda").manual_seed(0)
    hidden = torch.randn(T, H, device="cuda", generator=gen).bfloat16()
    w1 = (torch.randn(E, H, 2 * I, device="cuda", generator=gen) / H ** 0.5).bfloat16()
    w2 = (torch.randn(E, I, H, device="cuda", generator=gen) / I ** 0.5).bfloat16()
    wl, _ = B.make_workload(T, H, I, E, k, 1, rows=T * k)
    ws = B.Workspace(B.layer_workspace_size(wl))
    out, _ = B.layer_forward(hidden, B.pack_w1(w1), w2, r.expert_offsets, r.token_ids, r.gate_w, k, workspace=ws)
    assert ws.status() == 0
    y = torch.zeros(T * k, H, device="cuda", dtype=torch.bfloat16)
    x = X.dispatch_rows(hidden, r.slot_rows, T * k, out=torch.zeros_like(y))
    off = r.expert_offsets.tolist()
    for e in range(E):
        a, b = off[e], off[e + 1]
        h = x[a:b].float() @ w1[e].float()
        act = (torch.nn.functional.silu(h[:, :I]) * h[:, I:]).bfloat16()
        y[a:b] = (act.float() @ w2[e].float()).bfloat16()
    ref = X.combine_rows(y, r.slot_rows, gates)
    # two bf16 roundings on each side, each 2^-9 of its value at most
    assert (out - ref).norm() <= 4 * 2.0 ** -9 * ref.norm()
