"""Plain CPU oracle of the operators around and inside the experts, in numpy
and 64 bits: the sort of a router's choice, the rows' way to the experts and
back with its gradients, and microscaled 4-bit floating point with its product.
Test infrastructure: it shares no code with the library."""
import numpy as np

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def sort_by_expert(ids, gates, E, first=0):
    """offsets [E + 1], token_ids, gate_w [T topk] (then -1 and 0), slot_rows [T, topk]."""
    T, k = ids.shape
    rows = np.full((T, k), -1, np.int32)
    tok, gw = np.full(T * k, -1, np.int32), np.zeros(T * k, np.float32)
    off, at = np.zeros(E + 1, np.int32), 0
    for e in range(E):
        for t, j in np.argwhere(ids.astype(np.int64) == e + first):
            rows[t, j], tok[at], gw[at] = at, t, gates[t, j]
            at += 1
        off[e + 1] = at
    return off, tok, gw, rows


def _slots(slot_rows):
    for t, j in np.argwhere(slot_rows >= 0):
        yield t, j, slot_rows[t, j]


def dispatch(x, slot_rows, out):
    """Writes x's rows into out's and returns it (rows without a slot stay)."""
    for t, j, r in _slots(slot_rows):
        out[r] = x[t]
    return out


def combine(y, slot_rows, gates=None):
    """(sum, sum of magnitudes) [T, H] of each token's rows, weighted by gates if given."""
    out = np.zeros((slot_rows.shape[0], y.shape[1]))
    mag = np.zeros_like(out)
    for t, j, r in _slots(slot_rows):
        v = y[r].astype(np.float64) * (1.0 if gates is None else np.float64(gates[t, j]))
        out[t] += v
        mag[t] += np.abs(v)
    return out, mag


def combine_grad(dout, y, slot_rows, gates):
    """dy [rows, H] (0 for rows without a slot), dgates [T, topk] and the sum of
    the magnitudes of the latter's terms."""
    dy = np.zeros(y.shape)
    dg, mag = np.zeros(gates.shape), np.zeros(gates.shape)
    for t, j, r in _slots(slot_rows):
        dy[r] = np.float64(gates[t, j]) * dout[t]
        terms = y[r].astype(np.float64) * dout[t]
        dg[t, j], mag[t, j] = terms.sum(), np.abs(terms).sum()
    return dy, dg, mag


def mx4_quantize(x):
    """x [..., K] (64 bits) to (codes [..., KB, 32] of 0..15, scale bytes [..., KB])."""
    K = x.shape[-1]
    KB = -(-K // BLOCK)
    b = np.zeros(x.shape[:-1] + (KB * BLOCK,))
    b[..., :K] = x
    b = b.reshape(x.shape[:-1] + (KB, BLOCK))
    top = np.abs(b).max(-1)
    bad = ~np.isfinite(top)
    with np.errstate(all="ignore"):
        e = np.floor(np.log2(top)) - 2
    # log2 of a value just below a power of two may round up to it
    e = np.where(np.ldexp(1.0, np.where(np.isfinite(e), e, 0).astype(int) + 2) > top, e - 1, e)
    e = np.where(np.isfinite(e), np.maximum(e, -127), -127)
    with np.errstate(all="ignore"):
        v = np.minimum(np.abs(b) / np.exp2(e)[..., None], 6.0)
        d = np.abs(v[..., None] - GRID)
    # the nearest; of two equally near ones the even code
    lo = d.argmin(-1)
    hi = 7 - d[..., ::-1].argmin(-1)
    code = np.where(lo % 2 == 0, lo, hi) + 8 * np.signbit(b)
    return (np.where(bad[..., None], 0, code).astype(np.uint8),
            np.where(bad, 255, e + 127).astype(np.uint8))


def mx4_values(codes, scales):
    """Codes [..., KB, 32] and scale bytes [..., KB] as float64 [..., 32 KB]."""
    v = np.where(codes >= 8, -1.0, 1.0) * GRID[codes % 8]
    v = v * np.exp2(scales.astype(np.float64) - 127)[..., None]
    v = np.where(scales[..., None] == 255, np.nan, v)
    return v.reshape(v.shape[:-2] + (v.shape[-2] * v.shape[-1],))


def mx4_pack(codes, scales):
    """The layout in memory: two codes a byte, scale rows filled up to 4 bytes with zeros."""
    c = (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)
    pad = [(0, 0)] * (scales.ndim - 1) + [(0, -scales.shape[-1] % 4)]
    return c.reshape(c.shape[:-2] + (-1,)), np.pad(scales, pad)


def mx4_unpack(packed, scales):
    c = np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[:-1] + (-1, BLOCK))
    return c, scales[..., :c.shape[-2]]


def product(a, w, offsets, row_ids=None, swiglu=False):
    """a [A, K] and w [E, N, K] (64-bit values) to (out, sums of magnitudes)
    [rows, N]; with swiglu out [rows, N / 2] from gate columns, then up columns."""
    rows = int(offsets[-1])
    x = a[row_ids[:rows]] if row_ids is not None else a[:rows]
    y, mag = np.zeros((rows, w.shape[1])), np.zeros((rows, w.shape[1]))
    for e in range(len(offsets) - 1):
        s = slice(int(offsets[e]), int(offsets[e + 1]))
        y[s], mag[s] = x[s] @ w[e].T, np.abs(x[s]) @ np.abs(w[e]).T
    if not swiglu:
        return y, mag
    n = w.shape[1] // 2
    with np.errstate(over="ignore"):
        return y[:, :n] / (1 + np.exp(-y[:, :n])) * y[:, n:], mag
