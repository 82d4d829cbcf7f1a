"""Plain CPU oracle of what stands around the experts of a block, in numpy and 64
bits: the router's choice, the residual join with its norms and dropout, their
gradients, and the layer from the choice on.  Each returns what it computes and, for
comparisons, the sums of magnitudes that errors are relative to.  Test
infrastructure: it shares no code with the library."""
import numpy as np


def choose(logits, topk, bias=None, score="softmax", renormalize=True, scale=1.0):
    """ids [T, topk] and gates: logits as float32 values."""
    logits = np.asarray(logits, np.float32)
    T, E = logits.shape
    ids, gates = np.full((T, topk), -1, np.int32), np.zeros((T, topk))
    with np.errstate(all="ignore"):
        keys = logits if bias is None else logits + np.asarray(bias, np.float32)
    for t in range(T):
        k = [(-float(v), e) for e, v in enumerate(keys[t]) if v > -np.inf]
        for j, (_, e) in enumerate(sorted(k)[:topk]):
            ids[t, j] = e
        gates[t] = scores(logits[t].astype(np.float64), ids[t], score, renormalize, scale)
    return ids, gates


def scores(l, ids, score="softmax", renormalize=True, scale=1.0):
    """The gates of one token's chosen ids (-1: 0)."""
    on = ids >= 0
    out = np.zeros(len(ids))
    if not on.any():
        return out
    c = l[ids[on]]
    with np.errstate(all="ignore"):
        if score == "softmax":
            top = c.max() if renormalize else np.nanmax(l)
            p = np.exp(c - top)
            p = p / (p.sum() if renormalize else np.exp(l - top).sum())
        else:
            # (the logarithm of the sigmoid, so that a renormalised one never underflows)
            s = -np.logaddexp(0.0, -c)
            p = np.exp(s - s.max()) / np.exp(s - s.max()).sum() if renormalize else np.exp(s)
    out[on] = scale * p
    return out


def choose_grad(dgates, logits, ids, score="softmax", renormalize=True, scale=1.0):
    """dlogits [T, E] and the magnitudes of their terms."""
    l = np.asarray(logits, np.float64)
    dl, mag = np.zeros(l.shape), np.zeros(l.shape)
    for t in range(len(l)):
        q = scores(l[t], ids[t], score, renormalize)
        G, M = (q * dgates[t]).sum(), (q * np.abs(dgates[t])).sum()
        with np.errstate(all="ignore"):
            one = 1.0 / (1.0 + np.exp(l[t])) if score == "sigmoid" else np.ones(l.shape[1])   # 1 - p
        if score == "softmax" and not renormalize and (ids[t] >= 0).any():
            p = np.exp(l[t] - np.nanmax(l[t]))
            p /= p.sum()
            dl[t] -= scale * p * G
            mag[t] += scale * p * M
        for j, e in enumerate(ids[t]):
            if e < 0:
                continue
            g, m = dgates[t, j], abs(dgates[t, j])
            if renormalize:
                g, m = g - G, m + M
            dl[t, e] += scale * q[j] * one[e] * g
            mag[t, e] += scale * q[j] * one[e] * m
    return dl, mag


MASK = 2 ** 32 - 1


def philox(counter, key):
    """Philox4x32-10 in Python's integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & MASK, (a >> 32) ^ c[3] ^ k[1], a & MASK]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return c


def kept(seed, offset, T, H, p):
    """1 / (1 - p) where dropout keeps an element, else 0; p = 0: ones."""
    if p == 0.0:
        return np.ones((T, H))
    seed, offset = seed & (2 ** 64 - 1), offset & (2 ** 64 - 1)
    out = np.zeros((T, H))
    for t in range(T):
        for b in range((H + 3) // 4):
            w = philox((b, t, offset & MASK, offset >> 32), (seed & MASK, seed >> 32))
            for i in range(min(4, H - 4 * b)):
                out[t, 4 * b + i] = (1.0 / (1.0 - p)) if w[i] >= int(p * 2 ** 32) else 0.0
    return out


def _factor(x, eps):
    return 1.0 / np.sqrt((x * x).mean(1, keepdims=True) + eps)


def join(h, y, after=None, gate=None, scale=1.0, mask=1.0, eps=1e-6):
    """(x, scale times what is added) in 64 bits, x not rounded; h may be None."""
    a = y * _factor(y, eps) * after if after is not None else y
    a = scale * mask * (a if gate is None else a * gate)
    return (a if h is None else h + a), a


def norm(x, w, eps=1e-6):
    return x * _factor(x, eps) * w


def join_grad(dx, dz, x, y=None, after=None, gate=None, scale=1.0, mask=1.0, before=None, eps=1e-6):
    """Gradients {name: (value, bound of its terms' fp32 errors in units of 2^-24)}."""
    T, H = (dx if dx is not None else dz).shape
    out = {}
    d = np.zeros((T, H)) if dx is None else dx.astype(np.float64)
    tol = 2.0 * np.abs(d)
    if dz is not None:
        r, v = _factor(x, eps), dz * before
        d = d + r * (v - x * r * r * (x * v).mean(1, keepdims=True))
        tol = tol + 200.0 * r * (np.abs(v) + np.abs(x) * r * r * np.abs(x * v).mean(1, keepdims=True))
        out["before"] = ((dz * x * r).sum(0), (T + 64.0) * np.abs(dz * x * r).sum(0))
    out["h"] = (d, tol)
    if y is None:
        return out
    m = scale * mask
    da, tol = m * d, np.abs(m) * (tol + 4.0 * np.abs(d))
    q = _factor(y, eps) if after is not None else 1.0
    b = y * q * (after if after is not None else 1.0)
    if gate is not None:
        axis = 1 if gate.shape[0] == T and gate.shape != (1, H) else 0
        n = H if axis else T
        out["gate"] = ((da * b).sum(axis, keepdims=True),
                       (np.abs(b) * tol + (n + 64.0) * np.abs(da * b)).sum(axis, keepdims=True))
        da, tol = da * gate, np.abs(gate) * (tol + 2.0 * np.abs(da))
    if after is not None:
        out["after"] = ((da * y * q).sum(0), (np.abs(y * q) * tol + (T + 64.0) * np.abs(da * y * q)).sum(0))
        v = da * after
        tv = np.abs(after) * tol + np.abs(v)
        da = q * (v - y * q * q * (y * v).mean(1, keepdims=True))
        tol = q * (tv + np.abs(y) * q * q * (np.abs(y) * tv).mean(1, keepdims=True)
                   + 200.0 * (np.abs(v) + np.abs(y) * q * q * np.abs(y * v).mean(1, keepdims=True)))
    out["y"] = (da, tol)
    return out


def layer(x, w1, w2, ids, gates, first=0):
    """out [T, H] and how far it may be off, but for its own rounding: x [T, H], w1
    [E, H, 2I] (gate, then up columns), w2 [E, I, H].  An fp32 sum of n terms in any
    order is off by at most n 2^-24 of their magnitudes (twice that is allowed, since the
    matrix instruction adds in an order and with roundings of its own); the activation's
    two parts of bf16 are within 2^-8 2^-8 of it, its fp32 steps 16 2^-24, and below
    2^-126 a part may be lost; silu's slope is below 1.1."""
    T, H = x.shape
    E, I = w2.shape[0], w2.shape[1]
    u = 2.0 ** -24
    out, tol = np.zeros((T, H)), np.zeros((T, H))
    for t in range(T):
        for j in range(ids.shape[1]):
            e = int(ids[t, j]) - first
            if not 0 <= e < E:
                continue
            p = x[t] @ w1[e]
            tp = 2 * (H + 64) * u * (np.abs(x[t]) @ np.abs(w1[e]))
            g, up = p[:I], p[I:]
            with np.errstate(all="ignore"):
                s = g / (1.0 + np.exp(-g))
            a = s * up
            ta = 1.1 * tp[:I] * (np.abs(up) + tp[I:]) + np.abs(s) * tp[I:] + (16 * u + 2.0 ** -16) * np.abs(a) + 2.0 ** -126
            y = a @ w2[e]
            ty = ta @ np.abs(w2[e]) + 2 * (I + 64) * u * ((np.abs(a) + ta) @ np.abs(w2[e]))
            out[t] += gates[t, j] * y
            tol[t] += abs(gates[t, j]) * (ty + (ids.size + 64) * u * np.abs(y))
    return out, tol
