"""CPU: the kernels that 4-bit products run as, through a stand-in HIP runtime that
records launches (launch_recorder.py)."""
import pytest

import launch_recorder
import mx4_shapes

_PRODUCT = '''
vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
L.moe_mx4_product.argtypes = [vp] * 7 + [i64, i64, i32, i32, i32, i32, vp, vp]
def product(rows, K, N, E, swiglu, a_rows=100):
    """The kernel of a product, or the library's refusal."""
    r = L.moe_mx4_product(ADDR, ADDR, ADDR, ADDR, ADDR, ADDR, ADDR, a_rows, rows, K, N, E, swiglu, None, None)
    got = launches()
    assert len(got) == (r == 0), (r, got)
    return got[0] if got else r
'''


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    return launch_recorder.start(tmp_path_factory.mktemp("recorder"))


def test_the_shapes_reach_the_kernels_that_they_are_for(recorder):
    """Every kernel, with SwiGLU and without, over reductions, columns and experts:
    test_gpu_mx4_kernels.py compares each of these with the oracle."""
    shapes = [s for what in (mx4_shapes.REDUCTIONS, mx4_shapes.COLUMNS, mx4_shapes.EXPERTS) for s in mx4_shapes.shapes(what)]
    shapes += [(kernel, len(counts), K, N, rows) for kernel, counts, K, N, rows in mx4_shapes.SEVERAL]
    got = launch_recorder.run(recorder, _PRODUCT + f'''
result = [[product(rows, K, N, E, swiglu)[0] for swiglu in (0, 1) if swiglu == 0 or N % 2 == 0]
          for _, E, K, N, rows in {shapes}]
''')
    for (kernel, *shape), names in zip(shapes, got):
        for swiglu, name in zip(("false", "true"), names):
            assert name.startswith(f"{mx4_shapes.KERNELS[kernel]}, {swiglu}"), (shape, names)
    for what in (mx4_shapes.REDUCTIONS, mx4_shapes.COLUMNS, mx4_shapes.EXPERTS):
        assert len(what) == len(mx4_shapes.KERNELS)
