"""GPU: the post-router layer for a few tokens, in bf16 and with its weights in 4 bits,
against the 64-bit oracle (oracle/block.py derives how far it may be off)."""
import numpy as np
import pytest

from oracle import block as ob
from oracle import experts as oe

pytestmark = pytest.mark.gpu
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}


def _K():
    from paper_2609_07536_amd import block
    return block


def _bf16(a):
    import torch
    return torch.from_numpy(np.asarray(a)).bfloat16()


def _pack(w):
    """w1 [E, H, 2I] (gate, then up columns) as the up-projection reads it, on the GPU."""
    from paper_2609_07536_amd import binding
    return binding.pack_w1(w.cuda())


def _case(T, H, I, E, k, drop=0.0, seed=0, repeat=False):
    rng = np.random.default_rng([seed, T, H, I, E])
    ids = rng.integers(0, E, (T, k)) if repeat else np.argsort(rng.random((T, E)), 1)[:, :k]
    ids = ids.astype(np.int32)
    lost = rng.random((T, k)) < drop
    ids[lost] = rng.choice([-1, E, -2 ** 31, 2 ** 31 - 1], int(lost.sum()))
    gates = (rng.random((T, k)) * rng.choice([-1, 1], (T, k))).astype(np.float32)
    x = _bf16(rng.standard_normal((T, H)))
    w1 = _bf16(rng.standard_normal((E, H, 2 * I)) / H ** 0.5)
    w2 = _bf16(rng.standard_normal((E, I, H)) / I ** 0.5)
    return ids, gates, x, w1, w2


def _run(case, weights, dtype="float32", first=0):
    """layer_few into an output of NaN, with scratch of NaN bytes and no byte to spare."""
    import torch
    K = _K()
    ids, gates, x = case[:3]
    T, H = x.shape
    mx4 = isinstance(weights[1], tuple)
    I, E = (weights[1].K, weights[1].codes.shape[0]) if mx4 else (weights[1].shape[1], weights[1].shape[0])
    out = torch.full((T, H), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    n = K.layer_few_scratch_size(T, H, I, E, ids.shape[1])
    base = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")
    got = K.layer_few(x.cuda(), *weights, torch.from_numpy(ids).cuda(), torch.from_numpy(gates).cuda(),
                      first_expert=first, out=out, scratch=base[:n])
    assert bool((base[n:] == 255).all())
    return got.double().cpu().numpy()


def _check(got, case, w1, w2, dtype, first=0):
    ids, gates, x = case[:3]
    want, tol = ob.layer(x.double().numpy(), w1, w2, ids.astype(np.int64), gates.astype(np.float64), first)
    tol = tol + HALF[dtype] * (np.abs(want) + tol)
    assert (np.abs(got - want) <= tol).all()


CASES = [(1, 8, 16, 1, 1), (1, 512, 64, 8, 2), (2, 2048, 704, 32, 6), (3, 264, 48, 5, 3), (4, 40, 16, 4, 4), (5, 1352, 336, 11, 3),
         (7, 200, 80, 9, 2), (8, 1024, 256, 16, 8), (9, 72, 112, 40, 4), (12, 136, 32, 3, 3), (16, 1024, 512, 32, 8),
         (16, 56, 96, 100, 7), (16, 64, 16, 1, 1), (16, 32, 32, 1024, 64), (1, 32, 32, 64, 64), (13, 2048, 176, 30, 4)]


@pytest.mark.parametrize("T,H,I,E,k", CASES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_few_in_bf16(gpu_lib, T, H, I, E, k, dtype):
    case = _case(T, H, I, E, k, 0.15 if T > 2 else 0.0)
    got = _run(case, (_pack(case[3]), case[4].cuda()), dtype)
    _check(got, case, case[3].double().numpy(), case[4].double().numpy(), dtype)


def _mx4(w):
    """w [E, K, N] in MX4 [E, N, K], and the values that it stands for, [E, K, N]."""
    from paper_2609_07536_amd import experts as X
    codes, scales = oe.mx4_quantize(w.double().numpy().transpose(0, 2, 1))
    m = X.mx4_quantize_weights(w.cuda())
    return m, oe.mx4_values(codes, scales)[..., :w.shape[1]].transpose(0, 2, 1)


@pytest.mark.parametrize("T,H,I,E,k", CASES + [(1, 1, 1, 2, 1), (3, 33, 31, 4, 2), (6, 65, 7, 5, 5), (16, 257, 130, 9, 3),
                                               (2, 5, 100, 3, 2), (10, 999, 333, 12, 3), (4, 31, 33, 6, 2), (8, 127, 65, 8, 4)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_few_in_4_bits(gpu_lib, T, H, I, E, k, dtype):
    case = _case(T, H, I, E, k, 0.15 if T > 2 else 0.0)
    (m1, v1), (m2, v2) = _mx4(case[3]), _mx4(case[4])
    _check(_run(case, (m1, m2), dtype), case, v1, v2, dtype)


@pytest.mark.parametrize("mx4", [False, True])
def test_tokens_without_experts_and_experts_twice(gpu_lib, mx4):
    T, H, I, E, k = 11, 96, 48, 6, 4
    case = _case(T, H, I, E, k, 0.3, repeat=True)
    case[0][3] = -1
    case[0][5] = 2
    case[0][9, 1:] = case[0][9, 0]
    m1, m2 = _mx4(case[3]), _mx4(case[4])
    w1, w2 = (m1[1], m2[1]) if mx4 else (case[3].double().numpy(), case[4].double().numpy())
    weights = (m1[0], m2[0]) if mx4 else (_pack(case[3]), case[4].cuda())
    got = _run(case, weights)
    _check(got, case, w1, w2, "float32")
    assert not got[3].any()
    case[0][:] = -1
    assert not _run(case, weights).any()
    # the same bits again
    again = _case(T, H, I, E, k, 0.3, repeat=True)
    assert np.array_equal(_run(again, weights), _run(again, weights))


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("first", [0, 3, 1000, -2, 2 ** 31 - 5])
def test_a_share_of_the_experts(gpu_lib, mx4, first):
    T, H, I, E, k = 9, 64, 32, 5, 3
    case = _case(T, H, I, E, k)
    rng = np.random.default_rng(first % 1000)
    case[0][:] = np.clip(np.int64(first) + rng.integers(-2, E + 2, (T, k)), -2 ** 31, 2 ** 31 - 1)
    m1, m2 = _mx4(case[3]), _mx4(case[4])
    w1, w2 = (m1[1], m2[1]) if mx4 else (case[3].double().numpy(), case[4].double().numpy())
    _check(_run(case, (m1[0], m2[0]) if mx4 else (_pack(case[3]), case[4].cuda()), first=first), case, w1, w2, "float32", first)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("T", [3, 7, 16])
def test_infinities_and_nan_reach_their_own_tokens_alone(gpu_lib, mx4, T):
    """NaN in a token's row, in a gate that no expert takes, and in the weights of an
    expert that only one token names."""
    import torch
    H, I, E, k = 128, 64, 8, 2
    case = _case(T, H, I, E, k)
    ids, gates, x, w1, w2 = case
    ids[:] = np.arange(T)[:, None] % 5 + np.array([0, 1])
    ids[0] = [7, -1]
    gates[0, 1] = np.nan
    want = ob.layer(x.double().numpy(), w1.double().numpy(), w2.double().numpy(), ids.astype(np.int64),
                    np.nan_to_num(gates).astype(np.float64))
    x[1, 5] = float("nan")
    w1[7, 9, 3], w2[7, 2, :] = float("inf"), float("nan")
    if mx4:
        (m1, v1), (m2, v2) = _mx4(w1), _mx4(w2)
        with np.errstate(all="ignore"):
            want = ob.layer(x.double().numpy(), np.nan_to_num(v1), np.nan_to_num(v2), ids.astype(np.int64),
                            np.nan_to_num(gates).astype(np.float64))
    got = _run(case, (m1, m2) if mx4 else (_pack(w1), w2.cuda()))
    assert np.isnan(got[0]).all() and np.isnan(got[1]).all()
    assert (np.abs(got[2:] - want[0][2:]) <= (want[1] + 2.0 ** -24 * np.abs(want[0]))[2:]).all()


def test_few_agrees_with_the_layer(gpu_lib):
    """The layer of the sorted tokens, whose down-projection rounds its rows to bf16 as
    well: 2^-8 of them, and both within the oracle's bound."""
    import torch

    from paper_2609_07536_amd import binding as B
    from paper_2609_07536_amd import experts as X
    T, H, I, E, k = 16, 1024, 256, 16, 8
    ids, gates, x, w1, w2 = case = _case(T, H, I, E, k)
    packed, w = _pack(w1), w2.cuda()
    g = torch.from_numpy(gates).cuda()
    r = X.sort_by_expert(torch.from_numpy(ids).cuda(), g, E)
    out, _ = B.layer_forward(x.cuda(), packed, w, r.expert_offsets, r.token_ids, r.gate_w, k)
    got = _run(case, (packed, w))
    tol = ob.layer(x.double().numpy(), w1.double().numpy(), w2.double().numpy(), ids.astype(np.int64), gates.astype(np.float64))[1]
    rows = ob.layer(x.double().numpy(), w1.double().numpy(), w2.double().numpy(), ids.astype(np.int64), np.abs(gates).astype(np.float64))[0]
    # (each of the k rows is rounded; their magnitudes are below the bound's own sum over 2^-8)
    assert (np.abs(out.double().cpu().numpy() - got) <= 2 * tol + 2.0 ** -8 * k * np.abs(rows).max()).all()


def test_few_refuses_what_it_cannot_do(gpu_lib):
    import torch

    from paper_2609_07536_amd import binding as B
    K = _K()
    case = _case(16, 64, 32, 4, 2)
    w1, w2 = _pack(case[3]), case[4].cuda()
    x, ids, g = case[2].cuda(), torch.from_numpy(case[0]).cuda(), torch.from_numpy(case[1]).cuda()
    with pytest.raises(B.MoeError):      # 17 tokens
        K.layer_few(torch.cat([x, x[:1]]), w1, w2, torch.cat([ids, ids[:1]]), torch.cat([g, g[:1]]))
    with pytest.raises(B.MoeError):      # a scratch too small
        K.layer_few(x, w1, w2, ids, g, scratch=torch.empty(64, dtype=torch.uint8, device="cuda"))
    for bad in (lambda: K.layer_few(x.float(), w1, w2, ids, g), lambda: K.layer_few(x, w1, w2, ids.long(), g),
                lambda: K.layer_few(x, w1, w2, ids, g[:, :1]), lambda: K.layer_few(x, w1, w2.mT, ids, g),
                lambda: K.layer_few(x, w1[:, :, :16], w2, ids, g), lambda: K.layer_few(x, _mx4(case[3])[0], w2, ids, g)):
        with pytest.raises(TypeError):
            bad()
    e = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    assert K.layer_few(e, w1, w2, ids[:0], g[:0]).shape == (0, 64)
