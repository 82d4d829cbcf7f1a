"""CPU: the C ABI of the operators around and inside the experts - exports,
argument checks (nothing here launches work) - and the binding's refusals."""
import os
import re

import pytest
import torch

from paper_2609_07536_amd import binding as B
from paper_2609_07536_amd import experts as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_function():
    src = open(os.path.join(ROOT, "include", "moe_experts.h")).read()
    declared = set(re.findall(r"\b(moe_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", src, flags=re.S)))
    assert declared == set(X.EXPORTED)
    L = X.lib()
    assert all(hasattr(L, n) for n in declared) and L.moe_experts_abi_version() == 100


P = 1 << 20   # an aligned address that no refused call touches


def _sort(ids=P, gates=P, off=P, tok=P, gw=P, rows=P, T=10, k=2, E=4, first=0, scratch=None, nbytes=0):
    return X.lib().moe_sort_by_expert(ids, gates, off, tok, gw, rows, T, k, E, first, scratch, nbytes, None)


def test_sort_refusals():
    for bad in (dict(T=-1), dict(k=0), dict(E=0), dict(ids=None), dict(gates=None), dict(off=None), dict(tok=None),
                dict(gw=None), dict(rows=None)):
        assert _sort(**bad) == B.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(k=65), dict(E=1025), dict(T=2 ** 31 - 1, k=2), dict(T=2 ** 31 - 1, k=64)):
        assert _sort(**bad) == B.MOE_ERR_UNSUPPORTED, bad
    for bad in (dict(ids=P + 2), dict(gates=P + 1), dict(off=P + 2), dict(rows=P + 2), dict(scratch=P + 1)):
        assert _sort(**bad) == B.MOE_ERR_ALIGNMENT, bad
    need = X.sort_scratch_size(16384, 6, 32)
    assert 4 * 32 <= need <= 4 * 16384
    assert _sort(T=16384, k=6, E=32) == B.MOE_ERR_WORKSPACE
    assert _sort(T=16384, k=6, E=32, scratch=P, nbytes=need - 1) == B.MOE_ERR_WORKSPACE
    assert X.sort_scratch_size(512, 8, 1024) == 0 and X.sort_scratch_size(513, 8, 1024) >= 4 * 1024
    assert X.sort_scratch_size(10 ** 7, 8, 1024) <= 256 * 1024 * 4
    assert X.sort_scratch_size(-1, 8, 8) == X.sort_scratch_size(100000, 65, 8) == 0


def _rows(name, a=P, rows_in=P, b=P, T=10, k=2, rows=20, H=8, types=(0, 0), ws=None, gates=P, extra=P):
    L = X.lib()
    if name == "dispatch":
        return L.moe_dispatch_rows(a, rows_in, b, T, k, rows, H, ws, None)
    if name == "dispatch_grad":
        return L.moe_dispatch_rows_grad(a, rows_in, b, T, k, rows, H, *types, ws, None)
    if name == "combine":
        return L.moe_combine_rows(a, rows_in, gates, b, T, k, rows, H, *types, ws, None)
    return L.moe_combine_rows_grad(a, P, rows_in, gates, b, extra, T, k, rows, H, *types, ws, None)


@pytest.mark.parametrize("name", ["dispatch", "dispatch_grad", "combine", "combine_grad"])
def test_row_refusals(name):
    for bad in (dict(T=-1), dict(k=0), dict(rows=-1), dict(H=0), dict(rows_in=None), dict(a=None), dict(b=None)):
        assert _rows(name, **bad) == B.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(k=65), dict(rows=2 ** 31)):
        assert _rows(name, **bad) == B.MOE_ERR_UNSUPPORTED, bad
    for bad in (dict(rows_in=P + 2), dict(ws=P + 128)):
        assert _rows(name, **bad) == B.MOE_ERR_ALIGNMENT, bad
    if name != "dispatch":
        assert _rows(name, types=(2, 0)) == _rows(name, types=(0, -1)) == B.MOE_ERR_INVALID_ARG
        assert _rows(name, a=P + 1) == _rows(name, types=(1, 1), a=P + 2) == B.MOE_ERR_ALIGNMENT
    if name.startswith("combine"):
        assert _rows(name, gates=None) == B.MOE_ERR_INVALID_ARG
        assert _rows(name, gates=P + 2) == B.MOE_ERR_ALIGNMENT
    if name == "combine_grad":
        assert _rows(name, extra=None) == B.MOE_ERR_INVALID_ARG
    # nothing to do: no launch, no pointers needed
    assert _rows(name, T=0, a=None, b=None, rows_in=None, gates=None, extra=None) == B.MOE_OK


def test_binding_refusals():
    ids, g, x = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(4, 8)
    for call in (lambda: X.sort_by_expert(ids, g, 4), lambda: X.sort_by_expert(ids.long(), g, 4),
                 lambda: X.sort_by_expert(ids[0], g, 4), lambda: X.dispatch_rows(x, ids, 8),
                 lambda: X.dispatch_rows_grad(x, ids), lambda: X.combine_rows(x, ids, g),
                 lambda: X.combine_rows_grad(x, x, ids, g)):
        with pytest.raises(TypeError):
            call()


def _mx(name, a=P, b=P, c=P, rows=8, K=64, t=0, E=2, N=8):
    L = X.lib()
    if name == "weights":
        return L.moe_mx4_quantize_weights(a, b, c, E, K, N, t, None)
    if name == "quantize":
        return L.moe_mx4_quantize(a, b, c, rows, K, t, None)
    return L.moe_mx4_dequantize(b, c, a, rows, K, t, None)


@pytest.mark.parametrize("name", ["quantize", "weights", "dequantize"])
def test_mx4_refusals(name):
    for bad in (dict(K=0), dict(t=2), dict(t=-1), dict(a=None), dict(b=None), dict(c=None)):
        assert _mx(name, **bad) == B.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(K=2 ** 31 - 1), dict(K=2 ** 20, rows=2 ** 40, E=2 ** 15, N=2 ** 20)):
        assert _mx(name, **bad) == B.MOE_ERR_UNSUPPORTED, bad
    for bad in (dict(a=P + 1), dict(a=P + 2, t=1), dict(b=P + 8), dict(c=P + 2)):
        assert _mx(name, **bad) == B.MOE_ERR_ALIGNMENT, bad
    if name == "weights":
        assert _mx(name, E=0) == _mx(name, N=0) == B.MOE_ERR_INVALID_ARG
    else:
        assert _mx(name, rows=-1) == B.MOE_ERR_INVALID_ARG
        assert _mx(name, rows=0, a=None, b=None, c=None) == B.MOE_OK


def _product(a=P, s=P, w=P, ws=P, off=P, ids=P, out=P, a_rows=8, rows=16, K=64, N=8, E=2, swiglu=0, work=None):
    return X.lib().moe_mx4_product(a, s, w, ws, off, ids, out, a_rows, rows, K, N, E, swiglu, work, None)


def test_product_refusals():
    for bad in (dict(a=None), dict(s=None), dict(w=None), dict(ws=None), dict(off=None), dict(out=None), dict(a_rows=-1),
                dict(rows=-1), dict(K=0), dict(N=0), dict(E=0), dict(N=9, swiglu=1), dict(a_rows=0)):
        assert _product(**bad) == B.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(E=1025), dict(rows=2 ** 31), dict(a_rows=2 ** 31, K=32), dict(K=2 ** 20, N=2 ** 12)):
        assert _product(**bad) == B.MOE_ERR_UNSUPPORTED, bad
    for bad in (dict(a=P + 8), dict(s=P + 2), dict(w=P + 8), dict(ws=P + 1), dict(off=P + 2), dict(ids=P + 2),
                dict(out=P + 1), dict(work=P + 128)):
        assert _product(**bad) == B.MOE_ERR_ALIGNMENT, bad
    assert _product(rows=0, a=None, s=None, w=None, ws=None, off=None, ids=None, out=None) == B.MOE_OK


def _layer(h=P, w=P, off=P, rows_in=P, g=P, out=P, T=4, H=64, I=32, E=4, k=2, t=1, scratch=P, nbytes=1 << 30, ws=None):
    return X.lib().moe_mx4_layer_forward(h, w, P, P, P, off, P, rows_in, g, out, T, H, I, E, k, t, scratch, nbytes, ws,
                                         None)


def test_layer_refusals():
    for bad in (dict(h=None), dict(w=None), dict(off=None), dict(rows_in=None), dict(g=None), dict(out=None), dict(T=-1),
                dict(H=0), dict(I=0), dict(E=0), dict(k=0), dict(t=2)):
        assert _layer(**bad) == B.MOE_ERR_INVALID_ARG, bad
    for bad in (dict(k=65), dict(E=1025), dict(T=2 ** 30, k=4), dict(H=2 ** 20, I=2 ** 11)):
        assert _layer(nbytes=1 << 50, **bad) == B.MOE_ERR_UNSUPPORTED, bad
    need = X.mx4_layer_scratch_size(4, 64, 32, 2)
    assert need >= 4 * (32 + 4) + 8 * (64 + 16 + 4 + 128) and X.mx4_layer_scratch_size(4, 0, 32, 2) == 0
    for bad in (dict(scratch=None), dict(nbytes=need - 1)):
        assert _layer(**bad) == B.MOE_ERR_WORKSPACE, bad
    for bad in (dict(h=P + 1), dict(w=P + 8), dict(off=P + 2), dict(rows_in=P + 2), dict(g=P + 2), dict(out=P + 2),
                dict(scratch=P + 8), dict(ws=P + 128)):
        assert _layer(**bad) == B.MOE_ERR_ALIGNMENT, bad
    assert _layer(T=0, h=None, w=None, off=None, rows_in=None, g=None, out=None, scratch=None, nbytes=0) == B.MOE_OK


def test_oracle_by_hand():
    """The oracle against cases small enough to write down."""
    import numpy as np

    from oracle import experts as oe
    ids, gates = np.array([[1, 0], [-1, 1], [0, 5]], np.int32), np.arange(1, 7, dtype=np.float32).reshape(3, 2)
    off, tok, gw, rows = oe.sort_by_expert(ids, gates, 2)
    assert off.tolist() == [0, 2, 4] and tok.tolist() == [0, 2, 0, 1, -1, -1]
    assert gw.tolist() == [2, 5, 1, 4, 0, 0] and rows.tolist() == [[2, 0], [-1, 3], [1, -1]]
    x = np.zeros((3, 33))
    x[0, :5] = [6, 0.25, 0.75, -5, 2.5]      # 2^0: ties to the even code: 0, 1, -4, 2
    x[0, 32] = 2.0 ** -130                   # the least scale, 2^-127: rounds to 0
    x[1, :2] = [7, -1]                       # 2^0: 7 saturates to 6
    x[2, 1] = np.inf
    v = oe.mx4_values(*oe.mx4_quantize(x))
    assert v.shape == (3, 64) and v[0, :5].tolist() == [6, 0, 1, -4, 2] and v[0, 32] == 0
    assert v[1, :2].tolist() == [6, -1] and np.isnan(v[2, :32]).all() and (v[2, 32:] == 0).all()
