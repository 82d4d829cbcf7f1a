"""The operators of a mixture-of-experts block from the residual stream to the
residual stream, with their inputs, their plain forms and their definitions.

* ``choose``: a router's logits [T, E] to the experts and gates of each token,
  and ``choose_grad``, the gradient of the logits.
* ``join``: a block's output onto the residual stream (norm after the block,
  gate, dropout, residual scale) and the norm before the next block, in one pass,
  and ``join_grad``, the gradients of both streams, the norms' weights and the gate.
* ``few``: the whole post-router layer for up to 16 tokens, from the choice on,
  with weights in bf16 or in microscaled 4-bit floating point.

A program calls them for one token while it decodes for one user, for up to
tens of tokens in batched or speculative decoding, and (choose and join) for ten
thousand and more in prefill and training.  Routers score by softmax or
sigmoid, some with a bias that balances the load and acts on the choice alone;
``mask`` is the share of logits that are -inf (experts that a token may not take),
and with one one token in 16 may take none.
"""
import math

import numpy as np
import torch

own = False

# H, I, E, top-k: the repository's configurations, Granite's whole expert set, and odd sizes
SHAPES = {
    "tiny": dict(H=1024, I=512, E=8, topk=2),
    "granite": dict(H=1024, I=256, E=16, topk=8),
    "qwen": dict(H=2048, I=704, E=30, topk=4),
    "dsv2lite": dict(H=2048, I=704, E=32, topk=6),
    "granite_full": dict(H=1024, I=512, E=32, topk=8),
    "odd": dict(H=1352, I=336, E=11, topk=3),
}
EPS = 1e-6
BLOCK = 32


def _choose(name, T, E, topk, score="softmax", renorm=True, bias=False, mask=0.0, dtype="float32", scale=1.0, op="choose"):
    return dict(name=name, op=op, T=T, E=E, topk=topk, score=score, renorm=renorm, bias=bias, mask=mask, dtype=dtype,
                scale=scale)


def _join(name, T, H, h="bfloat16", y="float32", after=False, gate="none", scale=1.0, drop=0.0, before=True, op="join"):
    return dict(name=name, op=op, T=T, H=H, h=h, y=y, after=after, gate=gate, scale=scale, drop=drop, before=before)


def _few(name, shape, T, weights, drop=0.0):
    return dict(name=name, op="few", T=T, weights=weights, drop=drop, **SHAPES[shape])


def listed():
    return [
        # one user's decode step: one token's choice
        _choose("choose_decode_1", 1, 32, 6),
        # a prefill batch with a balanced sigmoid router of many experts
        _choose("choose_prefill_16384", 16384, 256, 8, "sigmoid", True, True, 0.0, "float32", 2.5),
        # the backward pass of a training step's softmax over all experts, some of them masked
        _choose("choose_grad_8192", 8192, 30, 4, "softmax", False, False, 0.05, op="choose_grad"),
        # one user's decode step: the layer's output onto the stream, the next block's norm
        _join("join_decode_1", 1, 2048),
        # a ragged chunk in training: norms on both sides, a gate for each token, dropout
        _join("join_ragged_777", 777, 1352, "bfloat16", "bfloat16", True, "token", 0.22, 0.1),
        # a prefill batch: the combine's fp32 output with a residual scale
        _join("join_prefill_16384", 16384, 2048, scale=0.22),
        # the backward pass of a training step
        _join("join_grad_8192", 8192, 2048, y="bfloat16", op="join_grad"),
        # the same with everything: both norms, a gate for each channel, dropout, odd sizes
        _join("join_grad_ragged_777", 777, 1351, "float32", "float32", True, "channel", 0.5, 0.2, op="join_grad"),
        # one user's decode step: six experts' weights read once
        _few("few_bf16_1", "dsv2lite", 1, "bf16"),
        # batched decoding of 16 sequences: nearly every expert's weights
        _few("few_bf16_16", "dsv2lite", 16, "bf16"),
        # one user's decode step with the weights in 4 bits
        _few("few_mx4_1", "dsv2lite", 1, "mx4"),
        # five drafted tokens through odd sizes, some slots without an expert
        _few("few_mx4_odd_5", "odd", 5, "mx4", 0.1),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(["choose", "choose_grad", "join", "join", "join_grad", "join_grad", "few", "few", "few"])
    if op.startswith("choose"):
        E = _log(rng, 2, 512)
        c = _choose("", min(_log(rng, 1, 16384), (1 << 22) // E), E, rng.randint(1, min(E, 8)),
                    rng.choice(["softmax", "sigmoid"]), rng.random() < 0.5, rng.random() < 0.3,
                    rng.choice([0.0, 0.0, 0.1, 0.5]), rng.choice(["float32", "bfloat16"]), rng.choice([1.0, 2.5]), op)
    elif op.startswith("join"):
        H = _log(rng, 48, 8192)
        c = _join("", min(_log(rng, 1, 16384), (1 << 24) // H), H, rng.choice(["bfloat16", "float32"]),
                  rng.choice(["bfloat16", "float32"]), rng.random() < 0.5, rng.choice(["none", "token", "channel"]),
                  rng.choice([1.0, 0.22]), rng.choice([0.0, round(rng.uniform(0.01, 0.6), 3)]), rng.random() < 0.8, op)
    else:
        c = _few("", rng.choice(sorted(SHAPES)), _log(rng, 1, 16), rng.choice(["bf16", "mx4"]), round(rng.uniform(0.01, 0.4), 3))
        if rng.random() < 0.4:   # sizes of no configuration (bf16 weights: H in eights, I in sixteens)
            c.update(H=8 * _log(rng, 16, 256), I=16 * _log(rng, 3, 44), E=_log(rng, 2, 48))
            c["topk"] = rng.randint(1, min(c["E"], 8))
            if c["weights"] == "mx4":
                c.update(H=c["H"] + rng.randint(0, 7), I=c["I"] + rng.randint(0, 15))
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------------

def _normal(shape, gen, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _empty(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _ids(case, seed):
    """A router's choice: topk different experts a token, a share of the slots without one."""
    g = np.random.default_rng([seed, case["T"], case["E"], case["topk"]])
    ids = np.argsort(g.random((case["T"], case["E"])), axis=1)[:, :case["topk"]].astype(np.int32)
    lost = g.random(ids.shape) < case["drop"]
    lost[0, 0] = False
    ids[lost] = -1
    return ids


def prepare(case, seed):
    """Inputs, and the buffers ("out", "scratch") that a program's loop keeps."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, st = case["op"], dict(case)
    if op.startswith("choose"):
        T, E, k = case["T"], case["E"], case["topk"]
        logits = _normal((T, E), gen, 1.5)
        if case["mask"]:
            logits[torch.rand((T, E), generator=gen, device="cuda") < case["mask"]] = -math.inf
            logits[torch.rand(T, generator=gen, device="cuda") < 1 / 16] = -math.inf
        st["logits"] = logits.to(getattr(torch, case["dtype"]))
        st["bias"] = _normal((E,), gen, 0.3) if case["bias"] else None
        if op == "choose":
            st["out"] = [_empty(T, k, dtype=torch.int32), _empty(T, k)]
        else:
            st["ids"] = _top(st["logits"].float(), st["bias"], k)[0].int()
            st["d"] = _normal((T, k), gen)
            st["out"] = torch.empty_like(st["logits"])
        return st
    if op.startswith("join"):
        T, H = case["T"], case["H"]
        th, ty = getattr(torch, case["h"]), getattr(torch, case["y"])
        st["h"] = _normal((T, H), gen, 2.0, th)      # the gradient's case: the stream after the join
        st["y"] = _normal((T, H), gen, 1.0, ty)
        st["w_after"] = 1 + _normal((H,), gen, 0.2) if case["after"] else None
        st["w_before"] = 1 + _normal((H,), gen, 0.2) if case["before"] else None
        shape = {"none": None, "token": (T, 1), "channel": (1, H)}[case["gate"]]
        st["g"] = torch.sigmoid(_normal(shape, gen)) if shape else None
        st["rng"] = torch.tensor([seed * 1000003 + 12345678901, seed * 7 + 5], device="cuda") if case["drop"] else None
        if op == "join":
            st["out"] = [_empty(T, H, dtype=th), _empty(T, H, dtype=torch.bfloat16) if case["before"] else None]
        else:
            st["d_h"] = _normal((T, H), gen, 1.0, th)
            st["d_z"] = _normal((T, H), gen, 1.0, torch.bfloat16) if case["before"] else None
            st["out"] = [_empty(T, H, dtype=th), _empty(T, H, dtype=ty), _empty(H) if case["after"] else None,
                         _empty(*shape) if shape else None, _empty(H) if case["before"] else None]
            st["scratch"] = _empty(1 << 25, dtype=torch.uint8)
        return st
    T, H, I, E, k = (case[n] for n in ("T", "H", "I", "E", "topk"))
    st["x"] = _normal((T, H), gen, 1.0, torch.bfloat16)
    st["ids"] = torch.from_numpy(_ids(case, seed)).cuda()
    st["gates"] = torch.softmax(_normal((T, k), gen), -1) * 2.0
    if case["weights"] == "bf16":
        st["w1"] = _normal((E, H, 2 * I), gen, 1.0 / math.sqrt(H), torch.bfloat16)   # packed, as the up-projection reads them
        st["w2"] = _normal((E, I, H), gen, 1.0 / math.sqrt(I), torch.bfloat16)
    else:
        # 4-bit codes and scales as a checkpoint brings them: [E, N, K], blocks of 32 along K
        for name, N, K in (("w1", 2 * I, H), ("w2", H, I)):
            kb = -(-K // BLOCK)
            codes = torch.randint(0, 256, (E, N, 16 * kb), generator=gen, device="cuda", dtype=torch.uint8)
            codes.view(E, N, kb, 16)[:, :, -1, (K - 32 * (kb - 1) + 1) // 2:] = 0
            if K % 2:
                codes[:, :, K // 2] &= 15
            scales = torch.zeros((E, N, kb + -kb % 4), device="cuda", dtype=torch.uint8)
            mean = 127 - int(round(math.log2(3.0 * math.sqrt(K))))
            scales[:, :, :kb] = torch.randint(mean - 1, mean + 2, (E, N, kb), generator=gen, device="cuda").to(torch.uint8)
            st[name + "_codes"], st[name + "_scales"] = codes, scales
    st["out"] = _empty(T, H, dtype=torch.bfloat16)
    st["scratch"] = _empty(1 << 22, dtype=torch.uint8)
    return st


# ---- the plain forms -----------------------------------------------------------------

def _top(logits, bias, k):
    """The experts of the k largest keys, ties to the lower index; -1 where a key is -inf or NaN."""
    key = logits if bias is None else logits + bias
    key = torch.where(torch.isnan(key), -math.inf, key)
    v, ids = torch.sort(key, dim=1, descending=True, stable=True)
    live = v[:, :k] > -math.inf
    return torch.where(live, ids[:, :k], -1), live


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _plain_choose(st):
    l = st["logits"].float()
    ids, live = _top(l, st["bias"], st["topk"])
    lc = l.gather(1, ids.clamp(min=0))
    if st["score"] == "softmax":
        if st["renorm"]:
            lc = torch.where(live, lc, -math.inf)
            top = lc.amax(1, keepdim=True)
            p = torch.where(live, torch.exp(lc - top), 0.0)
        else:
            top = l.amax(1, keepdim=True)
            p = torch.where(live, torch.exp(lc - top) / torch.exp(l - top).sum(1, keepdim=True), 0.0)
    else:
        p = torch.where(live, _sigmoid(lc), 0.0)
    if st["renorm"]:
        p = torch.where(live, p / p.sum(1, keepdim=True), 0.0)
    return [ids.int(), st["scale"] * p]


def _plain_choose_grad(st):
    l, ids, d = st["logits"].float(), st["ids"].long(), st["d"]
    live, at = ids >= 0, ids.clamp(min=0)
    lc = l.gather(1, at)
    dl = torch.zeros_like(l)
    if st["score"] == "softmax" and not st["renorm"]:
        p = torch.exp(l - l.amax(1, keepdim=True))
        p = torch.where(live.any(1, keepdim=True), p / p.sum(1, keepdim=True), 0.0)
        dl.scatter_add_(1, at, torch.where(live, d, 0.0))
        dl = st["scale"] * p * (dl - (p * dl).sum(1, keepdim=True))
        return dl.to(st["logits"].dtype)
    p = torch.where(live, torch.exp(lc - torch.where(live, lc, -math.inf).amax(1, keepdim=True))
                    if st["score"] == "softmax" else _sigmoid(lc), 0.0)
    if st["renorm"]:
        q = torch.where(live, p / p.sum(1, keepdim=True), 0.0)
        v = q * (d - (q * d).sum(1, keepdim=True))
        if st["score"] == "sigmoid":
            v = v * (1.0 - p)
    else:
        v = p * (1.0 - p) * d
    dl.scatter_add_(1, at, torch.where(live, st["scale"] * v, 0.0))
    return dl.to(st["logits"].dtype)


def _product32(a, m):
    """The high and low 32 bits of a * m (a: int64 values below 2^32)."""
    p = (a & 0xffff) * m
    q = (a >> 16) * m + (p >> 16)
    return q >> 16, ((q & 0xffff) << 16) | (p & 0xffff)


def _kept(rng, T, H, p):
    """Which elements dropout keeps [T, H]: Philox4x32-10 (Salmon et al., 2011), key the
    seed, counter (column / 4, row, offset), a word for each of four columns."""
    dev = rng.device
    lo, hi = rng & 0xffffffff, (rng >> 32) & 0xffffffff
    nb = -(-H // 4)
    c0 = torch.arange(nb, device=dev).expand(T, nb)
    c1 = torch.arange(T, device=dev)[:, None].expand(T, nb)
    c2, c3 = lo[1].expand(T, nb), hi[1].expand(T, nb)
    k0, k1 = lo[0], hi[0]
    for _ in range(10):
        h0, l0 = _product32(c0, 0xD2511F53)
        h1, l1 = _product32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return torch.stack([c0, c1, c2, c3], -1).view(T, 4 * nb)[:, :H] >= int(p * 2.0 ** 32)


def _rms(x):
    return torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)


def _plain_join(st):
    y, a = st["y"].float(), st["y"].float()
    if st["w_after"] is not None:
        a = y * _rms(y) * st["w_after"]
    if st["g"] is not None:
        a = a * st["g"]
    if st["drop"]:
        a = torch.where(_kept(st["rng"], st["T"], st["H"], st["drop"]), a / (1.0 - st["drop"]), 0.0)
    x = (st["h"].float() + st["scale"] * a).to(st["h"].dtype)
    if st["w_before"] is None:
        return [x]
    v = x.float()      # the norm of the stream as it is kept
    return [x, (v * _rms(v) * st["w_before"]).bfloat16()]


def _plain_join_grad(st):
    d, dbefore, dafter, dgate = st["d_h"].float(), None, None, None
    if st["w_before"] is not None:
        x, dz = st["h"].float(), st["d_z"].float()
        r = _rms(x)
        n = x * r
        dbefore = (dz * n).sum(0)
        v = dz * st["w_before"]
        d = d + r * (v - n * (v * n).mean(1, keepdim=True))
    da = st["scale"] * d
    if st["drop"]:
        da = torch.where(_kept(st["rng"], st["T"], st["H"], st["drop"]), da / (1.0 - st["drop"]), 0.0)
    y = st["y"].float()
    r = _rms(y) if st["w_after"] is not None else None
    b = y if r is None else y * r * st["w_after"]
    db = da
    if st["g"] is not None:
        dgate = (da * b).sum(1 if st["gate"] == "token" else 0, keepdim=True)
        db = da * st["g"]
    if r is not None:
        n = y * r
        dafter = (db * n).sum(0)
        v = db * st["w_after"]
        db = r * (v - n * (v * n).mean(1, keepdim=True))
    return [d.to(st["h"].dtype), db.to(st["y"].dtype), dafter, dgate, dbefore]


def _values(codes, scales, K):
    """fp32 [..., K] of 4-bit codes [..., 16 KB] (the lower half of a byte first) and scale bytes."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    grid = torch.cat([grid, -grid])
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    s = torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127)
    return (grid[c].unflatten(-1, (-1, BLOCK)) * s[..., :codes.shape[-1] // 16, None]).flatten(-2)[..., :K]


def _plain_few(st):
    T, k, H, I = st["T"], st["topk"], st["H"], st["I"]
    ids = st["ids"].reshape(-1).long()
    at, live = ids.clamp(min=0), ids >= 0
    x = st["x"].float().repeat_interleave(k, 0)[:, None]
    if st["weights"] == "bf16":
        p = torch.bmm(x, st["w1"][at].float())[:, 0].unflatten(1, (-1, 2, 16))
        g, u = p[:, :, 0].flatten(1), p[:, :, 1].flatten(1)
        y = torch.bmm((g * _sigmoid(g) * u)[:, None], st["w2"][at].float())[:, 0]
    else:
        p = (_values(st["w1_codes"][at], st["w1_scales"][at], H) * x).sum(2)
        g, u = p[:, :I], p[:, I:]
        y = (_values(st["w2_codes"][at], st["w2_scales"][at], I) * (g * _sigmoid(g) * u)[:, None]).sum(2)
    y = torch.where(live[:, None], y * st["gates"].reshape(-1, 1), 0.0)
    return y.view(T, k, H).sum(1).bfloat16()


# ---- one pass ------------------------------------------------------------------------

def run(st):
    op = st["op"]
    if not own:
        return {"choose": _plain_choose, "choose_grad": _plain_choose_grad, "join": _plain_join,
                "join_grad": _plain_join_grad, "few": _plain_few}[op](st)
    from paper_2609_07536_amd import block as K
    out = st["out"]
    if op == "choose":
        return list(K.choose(st["logits"], st["topk"], bias=st["bias"], score=st["score"], renormalize=st["renorm"],
                             scale=st["scale"], out=K.Choice(*out)))
    if op == "choose_grad":
        return K.choose_grad(st["d"], st["logits"], st["ids"], score=st["score"], renormalize=st["renorm"],
                             scale=st["scale"], out=out)
    if op == "join":
        r = K.join(st["h"], st["y"], after=st["w_after"], gate=st["g"], scale=st["scale"], drop=st["drop"],
                   rng=st["rng"], before=st["w_before"], eps=EPS, out=K.Joined(*out))
        return [r.h] if st["w_before"] is None else list(r)
    if op == "join_grad":
        return list(K.join_grad(st["d_h"], st["d_z"], st["h"], st["y"], after=st["w_after"], gate=st["g"],
                                scale=st["scale"], drop=st["drop"], rng=st["rng"], before=st["w_before"], eps=EPS,
                                out=K.JoinGrads(*out), scratch=st["scratch"]))
    if st["weights"] == "bf16":
        w1, w2 = st["w1"], st["w2"]
    else:
        from paper_2609_07536_amd.experts import MX4
        w1, w2 = MX4(st["w1_codes"], st["w1_scales"], st["H"]), MX4(st["w2_codes"], st["w2_scales"], st["I"])
    return K.layer_few(st["x"], w1, w2, st["ids"], st["gates"], out=out, scratch=st["scratch"])


def work(case):
    size = {"bfloat16": 2, "float32": 4}
    op, T = case["op"], case["T"]
    if op.startswith("choose"):
        n, s = T * case["E"] * size[case["dtype"]], 8 * T * case["topk"]
        return {"bytes": n * (1 if op == "choose" else 2) + s, "flops": 5 * T * case["E"]}
    if op.startswith("join"):
        H = case["H"]
        h, y, z = size[case["h"]], size[case["y"]], 2 if case["before"] else 0
        w = 4 * H * (case["after"] + case["before"] + (case["gate"] == "channel")) + (4 * T if case["gate"] == "token" else 0)
        if op == "join":
            return {"bytes": T * H * (2 * h + y + z) + w, "flops": 12 * T * H}
        return {"bytes": T * H * (2 * h + 2 * y + (z + h if z else 0)) + 2 * w, "flops": 24 * T * H}
    H, I, k = case["H"], case["I"], case["topk"]
    ids = _ids(case, 0)
    hit, slots = len(np.unique(ids[ids >= 0])), int((ids >= 0).sum())
    if case["weights"] == "bf16":
        weights = 6 * H * I
    else:
        weights = 17 * (2 * I * -(-H // BLOCK) + H * -(-I // BLOCK))
    return {"bytes": hit * weights + 4 * T * H + 8 * T * k, "flops": 6 * slots * H * I}


# ---- the definitions in 64 bits --------------------------------------------------------

def _exact_choose(st):
    l = st["logits"].double()
    k, T = st["topk"], st["T"]
    key = (st["logits"].float() + (0.0 if st["bias"] is None else st["bias"])).double()
    key = torch.nan_to_num(key, nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    ids = torch.argsort(-key, dim=1, stable=True)[:, :k] if st["op"] == "choose" else st["ids"].long().clamp(min=0)
    on = torch.zeros_like(l).scatter_(1, ids, 1.0) * (key > -math.inf)
    if st["op"] != "choose":
        on = torch.zeros_like(l)
        on[(torch.arange(T, device=l.device)[:, None].expand_as(ids))[st["ids"] >= 0], ids[st["ids"] >= 0]] = 1.0
    on = on > 0
    if st["score"] == "sigmoid":
        p = torch.special.expit(l)
    else:
        p = torch.nan_to_num(torch.softmax(l.masked_fill(~on, -math.inf) if st["renorm"] else l, 1), nan=0.0)
    q = p * on
    if st["renorm"] and st["score"] == "sigmoid":
        q = q / q.sum(1, keepdim=True).clamp(min=1e-300)
    return ids, on, p, q


def _dropped(rng, T, H, p):
    """1 / (1 - p) where an element is kept, 0 elsewhere, by 64-bit unsigned arithmetic on the host."""
    seed, offset = (int(v) & (2 ** 64 - 1) for v in rng.tolist())
    low = np.uint64(0xffffffff)
    nb = (H + 3) // 4
    ctr = [np.broadcast_to(np.arange(nb, dtype=np.uint64), (T, nb)),
           np.broadcast_to(np.arange(T, dtype=np.uint64)[:, None], (T, nb)),
           np.full((T, nb), offset & 0xffffffff, np.uint64), np.full((T, nb), offset >> 32, np.uint64)]
    for r in range(10):
        a, b = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ka = np.uint64(((seed & 0xffffffff) + r * 0x9E3779B9) & 0xffffffff)
        kb = np.uint64(((seed >> 32) + r * 0xBB67AE85) & 0xffffffff)
        ctr = [(b >> np.uint64(32)) ^ ctr[1] ^ ka, b & low, (a >> np.uint64(32)) ^ ctr[3] ^ kb, a & low]
    u = np.stack(ctr, 2).reshape(T, 4 * nb)[:, :H]
    return torch.from_numpy(np.where(u >= np.uint64(math.floor(p * 4294967296.0)), 1.0 / (1.0 - p), 0.0)).cuda()


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "choose":
        ids, on, _, q = _exact_choose(st)
        return [None, case["scale"] * q.gather(1, ids)]
    if op == "choose_grad":
        ids, on, p, q = _exact_choose(st)
        d = torch.zeros_like(p)
        d.scatter_add_(1, ids, torch.where(st["ids"] >= 0, st["d"].double(), 0.0))
        if case["score"] == "softmax":
            w = q if case["renorm"] else p * on.any(1, keepdim=True)
            return case["scale"] * w * (d - torch.linalg.vecdot(w, d)[:, None])
        if case["renorm"]:
            return case["scale"] * q * (1 - p) * (d - torch.linalg.vecdot(q, d)[:, None])
        return case["scale"] * q * (1 - p) * d
    if op.startswith("join"):
        T, H = case["T"], case["H"]
        m = _dropped(st["rng"], T, H, case["drop"]) if case["drop"] else 1.0
        m = m * case["scale"]
        g = 1.0 if st["g"] is None else st["g"].double()
        y = st["y"].double()
        ry = 1.0
        if st["w_after"] is not None:
            ry = 1.0 / torch.sqrt(torch.linalg.vecdot(y, y)[:, None] / H + EPS)
        wa = 1.0 if st["w_after"] is None else st["w_after"].double()
        if op == "join":
            x = st["h"].double() + m * g * (y * ry * wa)
            if st["w_before"] is None:
                return [x]
            v = x.to(st["h"].dtype).double()
            return [x, v * st["w_before"].double() / torch.sqrt(torch.linalg.vecdot(v, v)[:, None] / H + EPS)]
        d, dbefore, dafter, dgate = st["d_h"].double(), None, None, None
        if st["w_before"] is not None:
            x, v = st["h"].double(), st["d_z"].double() * st["w_before"].double()
            r = 1.0 / torch.sqrt(torch.linalg.vecdot(x, x)[:, None] / H + EPS)
            d = d + r * v - x * r ** 3 * torch.linalg.vecdot(v, x)[:, None] / H
            dbefore = torch.linalg.vecdot(st["d_z"].double().T, (x * r).T)
        da = m * d
        if st["g"] is not None:
            b = y * ry * wa
            dgate = torch.linalg.vecdot(da, b)[:, None] if case["gate"] == "token" else torch.linalg.vecdot(da.T, b.T)[None]
        db = da * g
        if st["w_after"] is not None:
            dafter = torch.linalg.vecdot(db.T, (y * ry).T)
            v = db * wa
            db = ry * v - y * ry ** 3 * torch.linalg.vecdot(v, y)[:, None] / H
        return [d, db, dafter, dgate, dbefore]
    out = torch.zeros((case["T"], case["H"]), dtype=torch.float64, device="cuda")
    H, I = case["H"], case["I"]
    table = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12, 0, -1, -2, -3, -4, -6, -8, -12], dtype=torch.float64, device="cuda") / 2

    def weights(name, e, K):
        c, s = st[name + "_codes"][e].long(), st[name + "_scales"][e].double()
        w = torch.empty((c.shape[0], 2 * c.shape[1]), dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = table[c % 16], table[c // 16]
        return (w * torch.exp2(s - 127)[:, :c.shape[1] // 16].repeat_interleave(BLOCK, 1))[:, :K].T
    for e in np.unique(_ids(case, seed)):
        if e < 0:
            continue
        t, j = torch.nonzero(st["ids"] == int(e), as_tuple=True)
        if case["weights"] == "bf16":
            w1, w2 = st["w1"][e].double().view(H, -1, 2, 16), st["w2"][e].double()
            wg, wu = w1[:, :, 0].reshape(H, I), w1[:, :, 1].reshape(H, I)
        else:
            w1, w2 = weights("w1", e, H), weights("w2", e, I)
            wg, wu = w1[:, :I], w1[:, I:]
        x = st["x"][t].double()
        y = torch.nn.functional.silu(x @ wg) * (x @ wu) @ w2
        out.index_add_(0, t, st["gates"][t, j].double()[:, None] * y)
    return out
