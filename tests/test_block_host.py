"""CPU: the C ABI of what stands around the experts - exports, argument checks
(nothing here launches work) -, the binding's refusals, and the oracle by hand and
against differences."""
import os
import re

import numpy as np
import pytest
import torch

from oracle import block as ob
from paper_2609_07536_amd import binding as B
from paper_2609_07536_amd import block as K
from paper_2609_07536_amd import experts as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20   # an aligned address that no refused call touches


def test_library_exports_every_declared_function():
    src = open(os.path.join(ROOT, "include", "moe_block.h")).read()
    declared = set(re.findall(r"\b(moe_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", src, flags=re.S)))
    assert declared == set(K.EXPORTED)
    L = K.lib()
    assert all(hasattr(L, n) for n in declared) and L.moe_block_abi_version() == 100
    assert re.search(r"#define MOE_FEW_TOKENS (\d+)", src).group(1) == str(K.FEW_TOKENS)


def _choose(name, logits=P, bias=None, ids=2 * P, gates=3 * P, T=10, E=8, k=2, t=0, score=0, out=4 * P, ws=None):
    L = K.lib()
    if name == "choose":
        return L.moe_choose(logits, bias, ids, gates, T, E, k, t, score, 1, 1.0, None)
    return L.moe_choose_grad(gates, logits, ids, out, T, E, k, t, score, 1, 1.0, ws, None)


@pytest.mark.parametrize("name", ["choose", "grad"])
def test_choose_refusals(name):
    for bad in (dict(T=-1), dict(E=0), dict(k=0), dict(k=9), dict(t=2), dict(t=-1), dict(score=2), dict(score=-1),
                dict(logits=None), dict(ids=None), dict(gates=None)):
        assert _choose(name, **bad) == B.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(E=1025), dict(E=100, k=65)):
        assert _choose(name, **bad) == B.MOE_ERR_UNSUPPORTED, bad
    for bad in (dict(logits=P + 1), dict(logits=P + 2, t=1), dict(ids=P + 2), dict(gates=P + 2)):
        assert _choose(name, **bad) == B.MOE_ERR_ALIGNMENT, bad
    if name == "choose":
        assert _choose(name, bias=P + 2) == B.MOE_ERR_ALIGNMENT
        for bad in (dict(ids=P), dict(gates=P), dict(ids=3 * P), dict(bias=3 * P), dict(bias=2 * P)):
            assert _choose(name, **bad) == B.MOE_ERR_INVALID_ARG, bad
    else:
        assert _choose(name, out=4 * P + 1) == _choose(name, ws=P + 128) == B.MOE_ERR_ALIGNMENT
        for bad in (dict(out=None), dict(out=P), dict(out=2 * P), dict(out=3 * P)):
            assert _choose(name, **bad) == B.MOE_ERR_INVALID_ARG, bad
    assert _choose(name, T=0, logits=None, ids=None, gates=None, out=None) == B.MOE_OK


def _join(h=P, y=2 * P, after=3 * P, gate=4 * P, before=5 * P, rng=6 * P, x=7 * P, z=8 * P, T=10, H=8, types=(0, 0, 0, 0),
          kind=1, drop=0.5):
    return K.lib().moe_join(h, y, after, gate, before, rng, x, z, T, H, *types, kind, 1.0, drop, 1e-6, None)


def test_join_refusals():
    bads = [dict(T=-1), dict(H=0), dict(kind=3), dict(kind=-1), dict(drop=1.0), dict(drop=-0.1), dict(drop=float("nan")),
            dict(gate=None), dict(rng=None), dict(h=None, y=None), dict(x=None), dict(z=None), dict(y=None),
            dict(y=None, after=None, gate=None, kind=0), dict(y=None, after=None, gate=None, kind=0, drop=0.0, before=None),
            dict(x=2 * P), dict(x=3 * P), dict(x=8 * P), dict(z=P), dict(z=2 * P), dict(z=5 * P), dict(x=6 * P),
            dict(x=P, y=P)]
    bads += [dict(types=t) for t in ((2, 0, 0, 0), (0, -1, 0, 0), (0, 0, 2, 0), (0, 0, 0, 2))]
    for bad in bads:
        assert _join(**bad) == B.MOE_ERR_INVALID_ARG, bad
    assert _join(H=16385) == B.MOE_ERR_UNSUPPORTED
    for bad in (dict(h=P + 1), dict(y=P + 1), dict(types=(1, 1, 1, 1), z=P + 2), dict(types=(0, 0, 0, 1), after=P + 2),
                dict(gate=P + 1), dict(before=P + 1), dict(rng=P + 4), dict(x=P + 1)):
        assert _join(**bad) == B.MOE_ERR_ALIGNMENT, bad
    assert _join(T=0) == B.MOE_OK


def _grad(dx=P, dz=2 * P, x=3 * P, y=4 * P, after=5 * P, gate=6 * P, before=7 * P, rng=8 * P, dh=9 * P, dy=10 * P,
          d_after=11 * P, d_gate=12 * P, d_before=13 * P, T=10, H=8, types=(0, 0, 0, 0), kind=2, drop=0.5, scratch=14 * P,
          room=1 << 30):
    return K.lib().moe_join_grad(dx, dz, x, y, after, gate, before, rng, dh, dy, d_after, d_gate, d_before, T, H, *types,
                                 kind, 1.0, drop, 1e-6, scratch, room, None)


def test_join_grad_refusals():
    bads = [dict(T=-1), dict(H=0), dict(kind=3), dict(drop=1.0), dict(gate=None), dict(rng=None), dict(dx=None, dz=None),
            dict(x=None), dict(before=None), dict(before=None, d_before=None), dict(y=None), dict(after=None),
            dict(kind=0), dict(dh=2 * P), dict(dh=3 * P), dict(dy=4 * P), dict(dy=P), dict(dy=9 * P), dict(d_after=5 * P),
            dict(d_after=12 * P), dict(d_before=7 * P), dict(d_before=12 * P), dict(dh=P, dz=P)]
    for bad in bads:
        assert _grad(**bad) == B.MOE_ERR_INVALID_ARG, bad
    assert _grad(H=16385) == B.MOE_ERR_UNSUPPORTED
    for bad in (dict(dx=P + 1), dict(dz=P + 1), dict(x=P + 1), dict(dh=P + 1), dict(dy=P + 1), dict(d_after=P + 2),
                dict(d_gate=P + 2), dict(d_before=P + 2), dict(scratch=P + 4)):
        assert _grad(**bad) == B.MOE_ERR_ALIGNMENT, bad
    need = K.join_grad_scratch_size(10, 8)
    assert need >= 3 * 4 * 8
    assert _grad(scratch=None) == _grad(room=need - 1) == B.MOE_ERR_WORKSPACE
    assert K.join_grad_scratch_size(-1, 8) == K.join_grad_scratch_size(8, 0) == K.join_grad_scratch_size(8, 16385) == 0
    assert K.join_grad_scratch_size(2 ** 40, 8) == 0
    assert _grad(T=0, d_after=None, d_gate=None, d_before=None) == B.MOE_OK


def _few(mx4, x=P, w1=2 * P, s1=3 * P, w2=4 * P, s2=5 * P, ids=6 * P, gates=7 * P, out=8 * P, T=2, H=64, I=32, E=4, k=2,
         first=0, t=0, scratch=9 * P, room=1 << 30):
    rest = (ids, gates, out, T, H, I, E, k, first, t, scratch, room, None)
    L = K.lib()
    return L.moe_few_forward_mx4(x, w1, s1, w2, s2, *rest) if mx4 else L.moe_few_forward(x, w1, w2, *rest)


@pytest.mark.parametrize("mx4", [False, True])
def test_few_refusals(mx4):
    for bad in (dict(T=-1), dict(H=0), dict(I=0), dict(E=0), dict(k=0), dict(t=2), dict(x=None), dict(w1=None),
                dict(w2=None), dict(ids=None), dict(gates=None), dict(out=None), dict(out=P), dict(out=2 * P),
                dict(out=9 * P), dict(out=7 * P)):
        assert _few(mx4, **bad) == B.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(T=17), dict(k=65), dict(E=1025), dict(H=1 << 23), dict(I=1 << 23), dict(H=1 << 20, I=1 << 16),
                dict(I=1 << 22, T=16, k=8, E=128)):
        assert _few(mx4, **bad) == B.MOE_ERR_UNSUPPORTED, bad
    for bad in (dict(x=P + 1), dict(w1=P + 8), dict(w2=P + 8), dict(ids=P + 2), dict(gates=P + 2), dict(out=P + 1),
                dict(out=P + 2, t=1), dict(scratch=P + 8)):
        assert _few(mx4, **bad) == B.MOE_ERR_ALIGNMENT, bad
    if mx4:
        assert _few(mx4, s1=None) == _few(mx4, s2=None) == B.MOE_ERR_INVALID_ARG
        assert _few(mx4, s1=P + 2) == _few(mx4, s2=P + 1) == B.MOE_ERR_ALIGNMENT
    else:
        assert _few(mx4, H=60) == _few(mx4, I=24) == B.MOE_ERR_UNSUPPORTED
    need = K.layer_few_scratch_size(2, 64, 32, 4, 2)
    assert need >= 2 * 4 * 32
    assert _few(mx4, scratch=None) == _few(mx4, room=need - 1) == B.MOE_ERR_WORKSPACE
    for bad in ((17, 64, 32, 4, 2), (2, 64, 0, 4, 2), (2, 64, 32, 4, 65), (2, 0, 32, 4, 2), (2, 64, 32, 1025, 2), (2 ** 40, 8, 8, 8, 8)):
        assert K.layer_few_scratch_size(*bad) == 0
    assert _few(mx4, T=0, x=None, ids=None, gates=None, out=None, scratch=None, room=0) == B.MOE_OK


def test_binding_refusals():
    l, ids, g, x = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(4, 8)
    w1, w2 = torch.zeros(2, 8, 32).bfloat16(), torch.zeros(2, 16, 8).bfloat16()
    for call in (lambda: K.choose(l, 2), lambda: K.choose(l[0], 2), lambda: K.choose_grad(g, l, ids), lambda: K.join(x, x),
                 lambda: K.join(None), lambda: K.join(x, before=x[0]), lambda: K.join_grad(x, None, x),
                 lambda: K.join_grad(None, x, None), lambda: K.layer_few(x.bfloat16(), w1, w2, ids, g)):
        with pytest.raises(TypeError):
            call()


def test_philox_known_answers():
    """The published known answers of Philox4x32-10 (zeros; all ones)."""
    assert ob.philox((0, 0, 0, 0), (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    f = 2 ** 32 - 1
    assert ob.philox((f, f, f, f), (f, f)) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


def test_choice_by_hand():
    inf, nan = np.inf, np.nan
    l = np.array([[1.0, 3.0, 3.0, 0.0], [-inf, nan, 2.0, -inf], [-inf] * 4, [0.0, -0.0, 0.0, -1.0]], np.float32)
    ids, gates = ob.choose(l, 3)
    assert ids.tolist() == [[1, 2, 0], [2, -1, -1], [-1, -1, -1], [0, 1, 2]]
    e = np.exp(-2.0)
    assert np.allclose(gates[0], np.array([1, 1, e]) / (2 + e)) and gates[1].tolist() == [1, 0, 0]
    assert gates[2].tolist() == [0, 0, 0] and np.allclose(gates[3], 1 / 3)
    # the bias acts on the choice alone
    ids, gates = ob.choose(l[:1], 2, np.array([5, 0, 0, 9]), "sigmoid", False, 2.0)
    assert ids.tolist() == [[3, 0]] and np.allclose(gates, 2 / (1 + np.exp([-0.0, -1.0])))
    # renormalised sigmoids far below underflow
    ids, gates = ob.choose(np.array([[-300.0, -301.0]], np.float32), 2, None, "sigmoid")
    assert np.allclose(gates, np.array([1, np.exp(-1)]) / (1 + np.exp(-1)))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_choice_gradient_against_differences(score, renorm):
    rng = np.random.default_rng(1)
    l = rng.standard_normal((3, 7))
    ids = np.array([[2, 5, 0], [6, -1, 1], [-1, -1, -1]])
    g = rng.standard_normal((3, 3))

    def f(l):
        return sum((ob.scores(l[t], ids[t], score, renorm, 1.7) * g[t]).sum() for t in range(3))
    got, _ = ob.choose_grad(g, l, ids, score, renorm, 1.7)
    for t in range(3):
        for e in range(7):
            d = np.zeros_like(l)
            d[t, e] = 1e-5
            assert abs((f(l + d) - f(l - d)) / 2e-5 - got[t, e]) < 1e-8


@pytest.mark.parametrize("kind", ["none", "token", "channel"])
@pytest.mark.parametrize("norms", [(True, True), (True, False), (False, True), (False, False)])
def test_join_gradient_against_differences(kind, norms):
    rng = np.random.default_rng(2)
    T, H = 3, 6
    h, y, cx, cz = (rng.standard_normal((T, H)) for _ in range(4))
    wa, wb = (rng.standard_normal(H) if n else None for n in norms)
    gate = {"none": None, "token": rng.standard_normal((T, 1)), "channel": rng.standard_normal((1, H))}[kind]
    mask = ob.kept(11, 5, T, H, 0.3)
    args = dict(h=h, y=y, after=wa, gate=gate, before=wb)

    def f(**kw):
        a = dict(args, **kw)
        x = ob.join(a["h"], a["y"], a["after"], a["gate"], 0.7, mask)[0]
        return (x * cx).sum() + ((ob.norm(x, a["before"]) * cz).sum() if wb is not None else 0.0)
    x = ob.join(h, y, wa, gate, 0.7, mask)[0]
    got = ob.join_grad(cx, cz if wb is not None else None, x, y, wa, gate, 0.7, mask, wb)
    for name, v in args.items():
        if v is None:
            continue
        for i in np.ndindex(v.shape):
            d = np.zeros_like(v)
            d[i] = 1e-5
            assert abs((f(**{name: v + d}) - f(**{name: v - d})) / 2e-5 - got[name][0][i]) < 1e-7, (name, i)


def test_a_gate_of_channels_is_needed_without_tokens_too():
    """Its H elements are read for the sums over no rows."""
    assert _grad(T=0, gate=None) == _join(T=0, gate=None, kind=2) == B.MOE_ERR_INVALID_ARG
    assert _join(T=0, gate=None) == B.MOE_OK


def test_a_differentiable_norm_alone_refuses_what_it_would_leave_out():
    from paper_2609_07536_amd import autograd as A
    x, w = torch.zeros(4, 8), torch.ones(8)
    for bad in (dict(before=w, gate=torch.ones(1, 8)), dict(before=w, after=w), dict(before=w, drop=0.5), dict()):
        with pytest.raises(TypeError):
            A.join(x, **bad)
    with pytest.raises(TypeError):
        A.join(None, before=w)


def test_join_grad_in_place_only_of_dx():
    """dh may be dx, and nothing else: also where dx has that other input's address.  (Without
    scratch no call gets past its checks.)"""
    inputs = dict(dz=2 * P, x=3 * P, y=4 * P, after=5 * P, gate=6 * P, before=7 * P, rng=8 * P)
    for name in inputs:
        assert _grad(dh=P, scratch=None, **{name: P}) == B.MOE_ERR_INVALID_ARG, name
        assert _grad(dx=inputs[name], dh=inputs[name], scratch=None) == B.MOE_ERR_INVALID_ARG, name
    assert _grad(dh=P, x=P, y=P, scratch=None) == B.MOE_ERR_INVALID_ARG
    assert _grad(dh=P, scratch=None) == B.MOE_ERR_WORKSPACE


def test_join_in_place_only_of_h():
    """x may be h, and nothing else: also where h has that other input's address."""
    for name in ("y", "after", "gate", "before", "rng"):
        assert _join(x=P, **{name: P}) == B.MOE_ERR_INVALID_ARG, name
        assert _join(z=P, **{name: P}) == B.MOE_ERR_INVALID_ARG, name


def test_scratch_of_the_most_rows_there_can_be():
    """2^31 - 1 rows fill the card's workgroups as 2^31 - 2 do; one of them would add up all
    rows alone."""
    for H in (1, 300, 16384):
        assert K.join_grad_scratch_size(2 ** 31 - 1, H) == K.join_grad_scratch_size(2 ** 31 - 2, H) > 0


def test_a_differentiable_join_with_dropout_refuses_to_go_without_numbers():
    from paper_2609_07536_amd import autograd as A
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        A.join(x, x, drop=0.5)
    with pytest.raises(TypeError):
        K.join(x, x, drop=0.5)


def test_join_grad_without_y_where_it_is_not_read():
    """With neither a norm after the block nor a gate dy says that the join had y.  (The calls
    that are taken get as far as their missing scratch.)"""
    plain = dict(y=None, after=None, gate=None, kind=0, d_after=None, d_gate=None, scratch=None)
    assert _grad(**plain) == B.MOE_ERR_WORKSPACE
    assert _grad(**plain, **{"drop": 0.0}) == B.MOE_ERR_WORKSPACE
    assert _grad(**{**plain, "dy": None}) == B.MOE_ERR_INVALID_ARG                 # dropout of nothing
    assert _grad(**{**plain, "after": 5 * P}) == B.MOE_ERR_INVALID_ARG
    assert _grad(**{**plain, "gate": 6 * P, "kind": 2}) == B.MOE_ERR_INVALID_ARG
    assert _grad(**{**plain, "gate": 6 * P, "kind": 1, "drop": 0.0}) == B.MOE_ERR_INVALID_ARG
    assert _grad(**{**plain, "dy": 10 * P + 1}) == B.MOE_ERR_ALIGNMENT
