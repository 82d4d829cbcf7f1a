"""GPU: the router's choice and the residual join with their gradients, against
the 64-bit oracle.

Tolerances, with u = 2^-24 (half a step of fp32) and half(t) = finfo(t).eps / 2:
* gates: exp is within 2 u of itself, its argument (a difference of logits, at most R
  in magnitude) is rounded once, which changes it by R u; sums of up to n positive
  terms are within n u, and a few further steps: (2 R + n + 16) u, relative.
* the gates' gradient: a product of a gate, whose error is that, and a difference of
  gradients (their weighted sum has topk terms).
* the join: a mean of squares is summed over at most 64 terms a lane, then lanes and
  waves: its relative error is below 96 u, the factor's (a root) below 52 u; each further
  step adds u; results are rounded to their type: half(t).
* the join's gradient: oracle/block.py carries each term's error along, in units of u.
"""
import numpy as np
import pytest

from oracle import block as ob

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}


def _K():
    from paper_2609_07536_amd import block
    return block


def _cuda(a, dtype=None, by=0):
    """On the GPU, `by` elements after an aligned address."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    t = t if dtype is None else t.to(getattr(torch, dtype))
    base = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")
    v = base[by:].view(t.shape)
    v.copy_(t)
    return v


def _f64(t):
    return None if t is None else t.double().cpu().numpy()


def _logits(seed, T, E, dtype, mask=0.0):
    import torch
    rng = np.random.default_rng(seed)
    l = rng.standard_normal((T, E)) * 2
    l[rng.random((T, E)) < mask] = -np.inf
    l[rng.random(T) < mask / 4] = -np.inf
    return rng, torch.from_numpy(l).to(getattr(torch, dtype)).float().numpy()


CHOICES = [(1, 1, 1), (1, 32, 6), (1, 2, 2), (7, 5, 3), (33, 11, 3), (64, 33, 8), (65, 64, 64), (100, 65, 4), (9, 128, 8),
           (50, 130, 7), (40, 256, 8), (11, 257, 6), (10, 512, 10), (5, 513, 64), (6, 1000, 5), (3, 1024, 64), (300, 30, 4)]


@pytest.mark.parametrize("T,E,k", CHOICES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("score,renorm,biased,mask", [("softmax", True, False, 0.0), ("softmax", False, True, 0.3),
                                                      ("sigmoid", True, True, 0.0), ("sigmoid", False, False, 0.9)])
def test_choose_and_its_gradient(gpu_lib, T, E, k, dtype, score, renorm, biased, mask):
    """bf16 logits are full of ties; masked ones leave slots, and tokens, without an expert."""
    import torch
    K = _K()
    rng, l = _logits([T, E, k], T, E, dtype, mask)
    bias = rng.standard_normal(E).astype(np.float32) if biased else None
    want, gates = ob.choose(l, k, bias, score, renorm, 1.5)
    dl = _cuda(l, dtype, 1)
    out = K.Choice(_cuda(np.full((T, k), 77, np.int32), by=1), _cuda(np.full((T, k), np.nan, np.float32), by=1))
    got = K.choose(dl, k, None if bias is None else _cuda(bias), score, renorm, 1.5, out=out)
    assert np.array_equal(got.expert_ids.cpu().numpy(), want)
    fin = l[np.isfinite(l)]
    R = float(fin.max() - fin.min()) if fin.size else 0.0
    rel = (2 * R + E + 16) * U
    assert (np.abs(_f64(got.gates) - gates) <= rel * np.abs(gates)).all()

    d = rng.standard_normal((T, k)).astype(np.float32)
    grad, mag = ob.choose_grad(d, l, want, score, renorm, 1.5)
    g = K.choose_grad(_cuda(d, by=1), dl, got.expert_ids, score, renorm, 1.5, out=_cuda(np.full((T, E), np.nan), dtype, 1))
    assert g.dtype == dl.dtype
    assert (np.abs(_f64(g) - grad) <= (2 * rel + (2 * k + 16) * U) * mag + HALF[dtype] * np.abs(grad)).all()


def test_choose_special_values(gpu_lib):
    """Equal keys go to the lower expert, -0 and 0 are equal, NaN and -inf are never chosen."""
    import torch
    K = _K()
    inf, nan = np.inf, np.nan
    l = np.array([[1.0, 3.0, 3.0, 0.0], [-inf, nan, 2.0, -inf], [-inf] * 4, [-0.0, 0.0, -0.0, -1.0], [nan] * 4,
                  [-100.0, -100.0, -200.0, -300.0], [3e38, -3e38, 0.0, 1.0]], np.float32)
    for score in ("softmax", "sigmoid"):
        want, gates = ob.choose(l, 3, None, score)
        got = K.choose(_cuda(l), 3, score=score)
        assert np.array_equal(got.expert_ids.cpu().numpy(), want)
        # (differences of logits up to 200 in the exponentials)
        assert (np.abs(_f64(got.gates) - gates) <= 450 * U * gates + 1e-38).all()
    bias = np.array([-inf, 0.0, nan, 1.0], np.float32)
    got = K.choose(_cuda(l[:1]), 4, _cuda(bias))
    assert got.expert_ids.tolist() == [[1, 3, -1, -1]] and got.gates[0, 2:].tolist() == [0.0, 0.0]


@pytest.mark.parametrize("score,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_choose_grad_of_ids_twice_and_of_bad_ids(gpu_lib, score, renorm):
    from paper_2609_07536_amd import binding as B
    K = _K()
    rng, l = _logits(5, 4, 20, "float32")
    ids = np.array([[3, 3, 7], [-1, 19, 19], [-1, -1, -1], [0, 5, 0]], np.int32)
    d = rng.standard_normal((4, 3)).astype(np.float32)
    grad, mag = ob.choose_grad(d, l, ids, score, renorm)
    ws = B.Workspace(512)
    got = K.choose_grad(_cuda(d), _cuda(l), _cuda(ids), score, renorm, workspace=ws)
    assert (np.abs(_f64(got) - grad) <= 200 * U * mag).all() and ws.status() == 0
    bad = np.where(ids == -1, np.array([20, -2, 2 ** 31 - 1], np.int32), ids)
    again = K.choose_grad(_cuda(d), _cuda(l), _cuda(bad), score, renorm, workspace=ws)
    assert np.array_equal(_f64(again), _f64(got)) and ws.status() == B.MOE_ERR_BAD_ROUTING


def test_choose_many_tokens(gpu_lib):
    """Every token of a large batch, against torch's stable sort."""
    import torch
    K = _K()
    l = torch.randn(200003, 60, device="cuda").bfloat16()
    got = K.choose(l, 8)
    v, ids = torch.sort(l.float(), dim=1, descending=True, stable=True)
    assert torch.equal(got.expert_ids, ids[:, :8].int())
    assert torch.allclose(got.gates, torch.softmax(v[:, :8].double(), -1).float(), rtol=64 * U, atol=0)


# ---- the join -------------------------------------------------------------------------

WIDTHS = [1, 2, 7, 8, 9, 48, 511, 512, 513, 1351, 1352, 2048, 2049, 4100, 8192, 8193, 16379, 16384]


def _join_case(T, H, h, y, gate, drop, seed=0, w="float32"):
    import torch
    rng = np.random.default_rng([T, H, seed])

    def rounded(a, t):
        return torch.from_numpy(np.asarray(a)).to(getattr(torch, t)).double().numpy()
    c = dict(h=rounded(rng.standard_normal((T, H)) * 2, h), y=rounded(rng.standard_normal((T, H)), y),
             after=rounded(1 + rng.standard_normal(H) / 4, w), before=rounded(1 + rng.standard_normal(H) / 4, w),
             gate={"none": None, "token": rounded(rng.standard_normal((T, 1)), w),
                   "channel": rounded(rng.standard_normal((1, H)), w)}[gate])
    c["rng"] = (int(rng.integers(-2 ** 63, 2 ** 63 - 1)), int(rng.integers(-2 ** 63, 2 ** 63 - 1)))
    c["mask"] = ob.kept(*c["rng"], T, H, drop)
    return rng, c


def _seeds(c):
    import torch
    return torch.tensor(c["rng"], dtype=torch.int64, device="cuda")


def _check_x(got, c, type_, scale, after, h=True):
    x, a = ob.join(c["h"] if h else None, c["y"], c["after"] if after else None, c["gate"], scale, c["mask"])
    tol = 64 * U * np.abs(a) + 2 * U * np.abs(x) + HALF[type_] * (np.abs(x) + 64 * U * np.abs(a))
    assert (np.abs(_f64(got) - x) <= tol).all()


def _check_z(got, x, w, type_):
    z = ob.norm(_f64(x), w)
    assert (np.abs(_f64(got) - z) <= (60 * U + HALF[type_] * (1 + 60 * U)) * np.abs(z)).all()


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("h,y,z,w", [("bfloat16", "float32", "bfloat16", "float32"), ("float32", "bfloat16", "float32", "bfloat16"),
                                     ("bfloat16", "bfloat16", "float32", "bfloat16"), ("float32", "float32", "bfloat16", "float32")])
@pytest.mark.parametrize("gate,after,drop", [("none", False, 0.0), ("token", True, 0.25), ("channel", True, 0.0),
                                             ("channel", False, 0.6)])
def test_join(gpu_lib, H, h, y, z, w, gate, after, drop):
    import torch
    K = _K()
    T, by = 5, H % 3
    _, c = _join_case(T, H, h, y, gate, drop, w=w)
    dh, dy = _cuda(c["h"], h, by), _cuda(c["y"], y, by)
    wa, wb = _cuda(c["after"], w, by) if after else None, _cuda(c["before"], w, by)
    g = _cuda(c["gate"], w, by) if c["gate"] is not None else None
    out = K.Joined(_cuda(np.full((T, H), np.nan), h, by), _cuda(np.full((T, H), np.nan), z, by))
    kw = dict(after=wa, gate=g, scale=0.75, drop=drop, rng=_seeds(c) if drop else None)
    r = K.join(dh, dy, before=wb, out=out, **kw)
    _check_x(r.h, c, h, 0.75, after)
    _check_z(r.z, r.h, c["before"], z)
    # without the norm before the next block; in place; with nothing to add to; the norm alone
    one = K.join(dh, dy, **kw)
    assert one.z is None and torch.equal(one.h, r.h)
    place = dh.clone()
    assert torch.equal(K.join(place, dy, out=K.Joined(place, None), **kw).h, r.h)
    alone = K.join(None, dy, **kw)
    assert alone.h.dtype == dy.dtype
    _check_x(alone.h, c, y, 0.75, after, h=False)
    norm = K.join(dh, before=wb, dtype=getattr(torch, z))
    assert norm.h is dh
    _check_z(norm.z, dh, c["before"], z)


@pytest.mark.parametrize("T,H", [(1, 2048), (3, 1), (1, 1), (700, 130), (2, 16384), (5, 8193), (9, 1351), (1100, 8), (4099, 33),
                                 (300, 2049), (30, 7), (1030, 513)])
@pytest.mark.parametrize("h,y,z,w", [("bfloat16", "float32", "bfloat16", "float32"), ("float32", "bfloat16", "float32", "bfloat16"),
                                     ("float32", "float32", "float32", "float32")])
@pytest.mark.parametrize("gate,after,before,drop", [("none", False, True, 0.0), ("token", True, True, 0.25),
                                                    ("channel", True, False, 0.0), ("channel", False, True, 0.5),
                                                    ("none", True, True, 0.1)])
def test_join_grad(gpu_lib, T, H, h, y, z, w, gate, after, before, drop):
    import torch
    K = _K()
    if drop and T * H > 200000:
        T = max(1, 200000 // H)     # (the oracle's random numbers are Python's)
    by = H % 3
    rng, c = _join_case(T, H, h, y, gate, drop, 1, w)
    dx, dz = (_cuda(rng.standard_normal((T, H)), t, by) for t in (h, z))
    dh, dy = _cuda(c["h"], h, by), _cuda(c["y"], y, by)
    wa, wb = _cuda(c["after"], w) if after else None, _cuda(c["before"], w) if before else None
    g = _cuda(c["gate"], w) if c["gate"] is not None else None
    kw = dict(after=wa, gate=g, scale=0.75, drop=drop, rng=_seeds(c) if drop else None, before=wb)
    for with_x, with_z in ((True, before), (False, True)):
        if not with_x and not before:
            continue
        want = ob.join_grad(_f64(dx) if with_x else None, _f64(dz) if with_z else None, c["h"], c["y"],
                            c["after"] if after else None, c["gate"], 0.75, c["mask"], c["before"])
        out = K.JoinGrads(*(None if t is None else torch.full_like(t, float("nan"), dtype=t.dtype if i < 2 else torch.float32)
                            for i, t in enumerate((dh, dy, wa, g, wb))))
        got = K.join_grad(dx if with_x else None, dz if with_z else None, dh, dy, out=out, **kw)
        for name, t in zip(K.JoinGrads._fields, got):
            if t is None:
                continue
            v, tol = want[name]
            t_type = {"h": h, "y": y}.get(name, "float32")
            tol = U * tol + HALF[t_type] * (np.abs(v) + U * tol)
            assert (np.abs(_f64(t).reshape(v.shape) - v) <= tol).all(), name
        # in place, only some of the outputs, and again: the same bits
        if with_x:
            place = dx.clone()
            again = K.join_grad(place, dz if with_z else None, dh, dy, out=K.JoinGrads(place, *[None] * 4), **kw)
            assert torch.equal(again.h, got.h)
        again = K.join_grad(dx if with_x else None, dz if with_z else None, dh, dy, residual=False, **kw)
        assert again.h is None
        for a, b in zip(again[1:], got[1:]):
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b))


def test_join_grad_of_a_norm_alone(gpu_lib):
    K = _K()
    rng, c = _join_case(37, 300, "float32", "float32", "none", 0.0)
    dz = rng.standard_normal((37, 300)).astype(np.float32)
    want = ob.join_grad(None, dz.astype(np.float64), c["h"], before=c["before"])
    got = K.join_grad(None, _cuda(dz), _cuda(c["h"], "float32"), before=_cuda(c["before"], "float32"))
    for name in ("h", "before"):
        v, tol = want[name]
        assert (np.abs(_f64(getattr(got, name)) - v) <= U * (tol + np.abs(v))).all()


def test_join_without_tokens(gpu_lib):
    import torch
    K = _K()
    e, w = torch.empty(0, 40, device="cuda"), torch.ones(40, device="cuda")
    r = K.join(e, e.bfloat16(), after=w, gate=torch.ones(1, 40, device="cuda"), before=w)
    assert r.h.shape == r.z.shape == (0, 40)
    out = K.JoinGrads(None, None, *(torch.full(s, 7.0, device="cuda") for s in ((40,), (1, 40), (40,))))
    got = K.join_grad(e, e, e, e, after=w, gate=w[None], before=w, out=out)
    assert all(not bool(t.any()) for t in got[2:])


def test_rows_of_infinities_and_nan_stay_in_their_rows(gpu_lib):
    import torch
    K = _K()
    x, w = torch.randn(6, 333, device="cuda"), torch.rand(333, device="cuda")
    y = x.flip(0).clone()
    want = K.join(x, y, after=w, before=w, dtype=torch.float32)
    y[2, 5], y[4, 7] = float("inf"), float("nan")
    got = K.join(x, y, after=w, before=w, dtype=torch.float32)
    for i in (0, 1, 3, 5):
        assert torch.equal(got.h[i], want.h[i]) and torch.equal(got.z[i], want.z[i])
    assert bool(got.z[2].isnan().any()) and bool(got.z[4].isnan().all())
    # zero rows: the norm of nothing is nothing
    assert not bool(K.join(torch.zeros(2, 9, device="cuda"), before=w[:9]).z.any())


def test_dropout_depends_on_seed_offset_row_and_column_alone(gpu_lib):
    import torch
    K = _K()
    x = torch.ones(50, 700, device="cuda")
    rng = torch.tensor([5, 9], device="cuda")
    a = K.join(None, x, drop=0.3, rng=rng).h
    assert torch.equal(a, K.join(None, x, drop=0.3, rng=rng).h)
    assert torch.equal(a[:20, :300], K.join(None, x[:20, :300].contiguous(), drop=0.3, rng=rng).h)
    for other in ([6, 9], [5, 10], [5 + 2 ** 32, 9], [5, 9 + 2 ** 32]):
        b = K.join(None, x, drop=0.3, rng=torch.tensor(other, device="cuda")).h
        # two independent masks agree on 0.58 of 35000 elements, give or take 0.0027
        assert abs(float((a == b).float().mean()) - 0.58) < 0.02
    # 35000 draws of probability 0.7 are within six standard deviations (0.0025) of it
    assert abs(float((a != 0).float().mean()) - 0.7) < 0.015
    # the gradient of a dropout is the same call on the gradient
    d = torch.randn_like(x)
    assert torch.equal(K.join_grad(d, None, None, x, drop=0.3, rng=rng, residual=False).y, K.join(None, d, drop=0.3, rng=rng).h)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_dropped_elements_take_nothing_from_an_infinite_gate(gpu_lib, dtype):
    """drop(a) is 0 where it drops, whatever a token's gate is: h goes on as it is there, to
    the bit, and what is kept is infinite."""
    import torch
    K = _K()
    T, H, p = 6, 700, 0.4
    rng = np.random.default_rng(5)
    h, y = _cuda(rng.standard_normal((T, H)), dtype), _cuda(rng.standard_normal((T, H)), dtype)
    gate = torch.ones(T, 1, device="cuda")
    gate[1], gate[4] = float("inf"), float("nan")
    kept = torch.from_numpy(ob.kept(3, 8, T, H, p) != 0).cuda()
    for y_h in (h, None):
        x = K.join(y_h, y, gate=gate, drop=p, rng=torch.tensor([3, 8], device="cuda")).h
        base = torch.zeros_like(y) if y_h is None else h
        assert torch.equal(x[~kept], base[~kept])
        assert bool(x[1][kept[1]].isinf().all()) and bool(x[4][kept[4]].isnan().all())
        assert bool(x[[0, 2, 3, 5]].isfinite().all())


def test_join_refuses_outputs_that_it_would_not_write(gpu_lib):
    """Without y the stream goes on in h, and without `before` there is no norm: a place for
    them would be returned as it was."""
    import torch
    K = _K()
    h, w = torch.randn(3, 40, device="cuda"), torch.rand(40, device="cuda")
    z, other = torch.empty_like(h), torch.full_like(h, 7.0)
    with pytest.raises(TypeError, match="out.h"):
        K.join(h, before=w, out=K.Joined(other, z))
    with pytest.raises(TypeError, match="out.z"):
        K.join(h, h.clone(), out=K.Joined(torch.empty_like(h), other))
    assert bool((other == 7.0).all())
    want = K.join(h, before=w, dtype=torch.float32)
    for place in (h, None, h.view(3, 40)):
        got = K.join(h, before=w, out=K.Joined(place, z))
        assert got.h.data_ptr() == h.data_ptr() and got.z is z and torch.equal(z, want.z)
