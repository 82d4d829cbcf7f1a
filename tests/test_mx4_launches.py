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


def test_calls_too_large_for_a_thin_kernel_run_as_tiles(recorder):
    """A thin kernel starts a workgroup for each of its tiles, and a launch has less than
    2^32 threads; the tiles' kernels take any number."""
    got = launch_recorder.run(recorder, _PRODUCT + """
result = [product(rows, K, N, E, 0) for rows, K, N, E in (
    ((1 << 30) + 5, 32, 2, 1), ((1 << 31) - 257, 32, 2, 1), ((1 << 31) - 257, 96, 33, 1000), (1 << 28, 32, 128, 1),
    (1 << 28, 32, 2, 1024), (1 << 29, 32, 2, 1), ((1 << 25) - 32, 32, 2, 1024))]
""")
    for call in got[:5]:
        assert "mx4_product_kernel" in call[0] and call[1] <= 512, call
    for call in got[5:]:
        assert "mx4_thin_kernel" in call[0] and call[1] * call[2] < 1 << 32, call
