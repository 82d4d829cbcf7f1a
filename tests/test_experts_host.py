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
