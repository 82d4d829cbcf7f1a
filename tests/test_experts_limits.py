"""CPU: the operators around the experts at the limits of their sizes: what does not fit
is refused, and what is launched near a limit covers it (nothing here runs on a GPU)."""
import types

import pytest
import torch

from paper_2609_07536_amd import binding as B
from paper_2609_07536_amd import experts as X

STREAM = types.SimpleNamespace(cuda_stream=0)
BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


class Tensor:
    """What the binding asks of a tensor, without memory."""
    is_cuda = True
    device = "cuda:0"

    def __init__(self, dtype, *shape):
        self.dtype, self.shape = dtype, torch.Size(shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def stride(self):
        return ()


def _mx4(*shape):
    codes, scales = X._mx4_shapes(shape[:-1], shape[-1])
    return X.MX4(Tensor(U8, *codes), Tensor(U8, *scales), shape[-1])


def _sort(T=4, k=2, E=8, first=0):
    n = T * k
    out = X.Routing(Tensor(I32, E + 1), Tensor(I32, n), Tensor(F32, n), Tensor(I32, T, k))
    return X.sort_by_expert(Tensor(I32, T, k), Tensor(F32, T, k), E, first, out=out, scratch=Tensor(U8, 1 << 40), stream=STREAM)


def _rows(name, T=4, k=2, rows=8, H=16):
    slots, gates, y, x = Tensor(I32, T, k), Tensor(F32, T, k), Tensor(F32, rows, H), Tensor(F32, T, H)
    if name == "dispatch":
        return X.dispatch_rows(x, slots, rows, out=y, stream=STREAM)
    if name == "dispatch_grad":
        return X.dispatch_rows_grad(y, slots, out=x, stream=STREAM)
    if name == "combine":
        return X.combine_rows(y, slots, gates, out=x, stream=STREAM)
    return X.combine_rows_grad(x, y, slots, gates, out=(y, gates), stream=STREAM)


def _product(E=4, N=8, K=64, rows=0):
    return X.mx4_product(_mx4(rows, K), _mx4(E, N, K), Tensor(I32, E + 1), rows, out=Tensor(BF16, rows, N), stream=STREAM)


def _layer(T=0, H=64, I=32, E=4, k=2):
    r = X.Routing(Tensor(I32, E + 1), Tensor(I32, T * k), Tensor(F32, T * k), Tensor(I32, T, k))
    return X.layer_forward_mx4(Tensor(BF16, T, H), _mx4(E, 2 * I, H), _mx4(E, H, I), r, Tensor(F32, T, k),
                               out=Tensor(F32, T, H), scratch=Tensor(U8, 1 << 40), stream=STREAM)


BIG = 2 ** 32   # (of BIG + n, 32 bits keep n)


@pytest.mark.parametrize("call", [
    lambda: _sort(T=BIG), lambda: _sort(T=BIG + 4), lambda: _sort(T=0, k=BIG + 2), lambda: _sort(E=BIG + 8), lambda: _sort(T=0, E=2 ** 31),
    lambda: _sort(first=2 ** 31), lambda: _sort(first=-2 ** 31 - 1), lambda: _sort(first=BIG),
    *[lambda n=n, kw=kw: _rows(n, **kw) for n in ("dispatch", "dispatch_grad", "combine", "combine_grad")
      for kw in (dict(T=BIG), dict(T=0, k=BIG + 2), dict(T=0, rows=2 ** 31))],
    *[lambda n=n: _rows(n, T=0, rows=0, H=BIG + 16) for n in ("dispatch", "dispatch_grad", "combine", "combine_grad")],
    lambda: X.mx4_quantize(Tensor(F32, 0, BIG + 64), out=_mx4(0, BIG + 64), stream=STREAM),
    lambda: X.mx4_dequantize(_mx4(0, BIG + 64), out=Tensor(F32, 0, BIG + 64), stream=STREAM),
    *[lambda s=s: X.mx4_quantize_weights(Tensor(F32, *s), out=_mx4(s[0], s[2], s[1]), stream=STREAM)
      for s in ((BIG + 1, 64, 8), (1, BIG + 64, 8), (1, 64, BIG + 8))],
    lambda: _product(E=BIG + 4), lambda: _product(N=BIG + 8), lambda: _product(K=BIG + 64), lambda: _product(rows=2 ** 31),
    lambda: _layer(T=BIG), lambda: _layer(H=BIG + 64), lambda: _layer(I=BIG + 32), lambda: _layer(E=BIG + 4),
    lambda: _layer(k=BIG + 2)])
def test_sizes_past_32_bits_are_refused_by_the_binding(call):
    """They are not cut to the 32 bits that the library takes."""
    with pytest.raises(B.MoeError) as e:
        call()
    assert e.value.code == B.MOE_ERR_UNSUPPORTED


def test_sizes_of_scratch_past_32_bits():
    """0, as for every invalid argument."""
    assert X.sort_scratch_size(BIG + 16384, 6, 32) == X.sort_scratch_size(16384, 6, BIG + 32) == 0
    assert X.sort_scratch_size(16384, BIG + 6, 32) == 0
    for big in ((BIG + 4, 64, 32, 2), (4, BIG + 64, 32, 2), (4, 64, BIG + 32, 2), (4, 64, 32, BIG + 2)):
        assert X.mx4_layer_scratch_size(*big) == 0


P = 1 << 20   # an aligned address that no refused call touches


def test_columns_near_2_to_31():
    """Past what the kernels' 32-bit steps over the columns hold (a loop over 2048 of
    them at a time passes 2^31 - 1 before it ends)."""
    L = X.lib()
    for H, code in ((2 ** 31 - 1, B.MOE_ERR_UNSUPPORTED), (2 ** 31 - 4096, B.MOE_ERR_UNSUPPORTED), (0, B.MOE_ERR_INVALID_ARG)):
        assert L.moe_dispatch_rows_grad(P, P, P, 1, 1, 1, H, 0, 0, None, None) == code
        assert L.moe_combine_rows(P, P, P, P, 1, 1, 1, H, 0, 0, None, None) == code
        assert L.moe_combine_rows_grad(P, P, P, P, P, P, 1, 1, 1, H, 0, 0, None, None) == code


def test_elements_of_the_quantisers_near_their_limits():
    """Columns of weights past what tiles of 128 count in 32 bits, and a launch of 2^32
    threads, which the runtime has no room for."""
    L = X.lib()
    for N in (2 ** 31 - 1, 2 ** 31 - 256):
        assert L.moe_mx4_quantize_weights(P, P, P, 1, 1, N, 0, None) == B.MOE_ERR_UNSUPPORTED
    assert L.moe_mx4_quantize_weights(P, P, P, 2 ** 24, 1, 1, 0, None) == B.MOE_ERR_UNSUPPORTED
    for rows, K in ((2 ** 30, 32), (2 ** 20, 2 ** 15)):   # 2^35 elements, eight a thread
        assert L.moe_mx4_quantize(P, P, P, rows, K, 0, None) == B.MOE_ERR_UNSUPPORTED
        assert L.moe_mx4_dequantize(P, P, P, rows, K, 0, None) == B.MOE_ERR_UNSUPPORTED


def test_rows_and_reduction_of_a_product_near_2_to_31():
    """Rounded up to whole tiles and blocks they pass 32 bits."""
    L = X.lib()

    def product(rows=16, K=64, N=1, a_rows=1):
        return L.moe_mx4_product(P, P, P, P, P, P, P, a_rows, rows, K, N, 1, 0, None, None)
    for n in (2 ** 31 - 1, 2 ** 31 - 256):
        assert product(rows=n) == product(K=n) == B.MOE_ERR_UNSUPPORTED
    assert L.moe_mx4_layer_forward(*[P] * 10, 2 ** 31 - 256, 64, 64, 4, 1, 1, P, 1 << 60, None, None) == B.MOE_ERR_UNSUPPORTED


def test_slots_that_a_sort_takes_without_scratch():
    """The binding's constant is the library's."""
    n = X._SORT_WITHOUT_SCRATCH
    for E in (1, 32, 1024):
        assert X.sort_scratch_size(n, 1, E) == 0 < X.sort_scratch_size(n + 1, 1, E)


def test_an_output_in_place_of_an_input_is_refused():
    """Other tokens' rows may still have to be read.  (combine's dy may be its y: each row
    is read and written by its own slot's wave.)"""
    L, Q = X.lib(), P + (1 << 16)
    assert L.moe_dispatch_rows(P, Q, P, 4, 1, 4, 32, None, None) == B.MOE_ERR_INVALID_ARG
    assert L.moe_dispatch_rows_grad(P, Q, P, 4, 1, 4, 32, 1, 1, None, None) == B.MOE_ERR_INVALID_ARG
    assert L.moe_combine_rows(P, Q, Q, P, 4, 1, 4, 32, 1, 1, None, None) == B.MOE_ERR_INVALID_ARG
    assert L.moe_combine_rows_grad(P, Q, Q, Q, P, Q, 4, 1, 4, 32, 1, 1, None, None) == B.MOE_ERR_INVALID_ARG


def test_slots_of_a_sort_near_2_to_31():
    L = X.lib()
    for T, k in ((2 ** 31 - 2 ** 24, 1), (2 ** 26, 32)):
        assert L.moe_sort_by_expert(P, P, P, P, P, P, T, k, 8, 0, P, 1 << 40, None) == B.MOE_ERR_UNSUPPORTED
        assert X.sort_scratch_size(T, k, 8) == 0
    assert X.sort_scratch_size(2 ** 31 - 2 ** 24 - 1, 1, 8) == 256 * 8 * 4
