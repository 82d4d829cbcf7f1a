"""GPU: the operators around the experts where sizes and offsets pass 31 and 32 bits."""
import numpy as np
import pytest

from oracle import experts as oe

pytestmark = pytest.mark.gpu


def test_row_ids_past_4_gib(gpu_lib):
    """A gathered product of 2^30 + 4999 rows (ids past 2^32 bytes, 137 GB of output): rows
    around 2^29 and 2^30 and the last ones against the oracle."""
    import torch

    from paper_2609_07536_amd import binding as B
    from paper_2609_07536_amd import experts as X
    K, N, A, M = 32, 128, 500, (1 << 30) + 4999
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("needs 160 GiB of free GPU memory")
    gen = torch.Generator(device="cuda").manual_seed(0)
    a = X.mx4_quantize(torch.randn(A, K, device="cuda", generator=gen))
    w = X.mx4_quantize_weights(torch.randn(2, K, N, device="cuda", generator=gen) / 4)
    ids = torch.randint(0, A, (M,), dtype=torch.int32, device="cuda", generator=gen)
    first = (1 << 30) - 100
    off = torch.tensor([0, first, M], dtype=torch.int32, device="cuda")
    out = torch.empty(M, N // 2, dtype=torch.bfloat16, device="cuda")
    ws = B.Workspace(512)
    X.mx4_product(a, w, off, M, row_ids=ids, swiglu=True, out=out, workspace=ws)
    assert ws.status() == 0
    va, vw = (X.mx4_dequantize(m, dtype=torch.float32).double().cpu().numpy() for m in (a, w))
    for r0, r1 in ((0, 130), ((1 << 29) - 200, (1 << 29) + 200), (first - 130, (1 << 30) + 130), (M - 300, M)):
        split = min(max(first - r0, 0), r1 - r0)
        got = out[r0:r1].double().cpu().numpy()
        where = ids[r0:r1].cpu().numpy()
        y, S = oe.product(va, vw, np.array([0, split, r1 - r0]), where)
        want = oe.product(va, vw, np.array([0, split, r1 - r0]), where, True)[0]
        g, u = y[:, :N // 2], y[:, N // 2:]
        d = K * 2.0 ** -24 * np.maximum(S[:, :N // 2], S[:, N // 2:])
        silu = g / (1 + np.exp(-g))
        tol = (1.1 * np.abs(u) + np.abs(silu) + d) * d + 2 * 2.0 ** -8 * np.abs(want)
        assert (np.abs(got - want) <= tol).all(), (r0, r1)
    del out, ids
    torch.cuda.empty_cache()


def test_rows_of_a_large_tensor_each_in_their_place(gpu_lib):
    """Quantised and back, 2.6e9 elements: rows on either side of 2^31 elements and the last
    ones hold values of their own, all others zeros."""
    import torch

    from paper_2609_07536_amd import experts as X
    rows, K = 40000, 65536
    where = [0, 1, 7231, 7232, 32767, 32768, 32769, 39998, 39999]   # (7232 = 40000 - 2^31 / K)
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    x[where] = torch.randn(len(where), K, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0)).bfloat16()
    q = X.mx4_quantize(x)
    codes, scales = oe.mx4_quantize(x[where].double().cpu().numpy())
    packed = oe.mx4_pack(codes, scales)
    assert np.array_equal(q.codes[where].cpu().numpy(), packed[0]) and np.array_equal(q.scales[where].cpu().numpy(), packed[1])
    back = torch.full_like(x, 9.0)
    X.mx4_dequantize(q, out=back)
    assert np.array_equal(back[where].double().cpu().numpy(), oe.mx4_values(codes, scales))
    back[where] = 0
    assert not bool(back.any())
    q.codes[where] = 0
    assert not bool(q.codes.any())


@pytest.mark.parametrize("H", [1, 7, 9, 511, 513, 2049, 4100])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_combine_gradient_in_place_of_its_rows(gpu_lib, H, dtype):
    """dy written over y: the same, bit for bit, as beside it."""
    import torch

    from paper_2609_07536_amd import experts as X
    T, k, E = 300, 3, 8
    gen = torch.Generator(device="cuda").manual_seed(H)
    ids = torch.randint(-1, E, (T, k), dtype=torch.int32, device="cuda", generator=gen)
    gates = torch.randn(T, k, device="cuda", generator=gen)
    r = X.sort_by_expert(ids, gates, E)
    y = torch.randn(T * k, H, device="cuda", generator=gen).to(getattr(torch, dtype))
    d = torch.randn(T, H, device="cuda", generator=gen)
    live = int(r.expert_offsets[-1])
    dy, dg = X.combine_rows_grad(d, y, r.slot_rows, gates)
    got, dg2 = X.combine_rows_grad(d, y, r.slot_rows, gates, out=(y, torch.empty_like(gates)))
    assert got is y and torch.equal(y[:live], dy[:live]) and torch.equal(dg2, dg)
