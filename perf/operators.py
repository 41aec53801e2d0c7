"""The work that the transformer operators over voxel features are timed on.

A case is a dict of plain values.  Its ``kind`` names the operator that one pass runs:

  norm     root-mean-square norm of rows, with the residual's addition, and with its result
           in the rows' type or in 8 bits (e4m3) with a scale for each 128 columns
  linear   product of 8-bit rows and 8-bit weights, scaled by blocks of 128, with ReLU
  attend   attention inside the documents (scenes) of a packed batch: queries aligned with
           the end of their document's keys, shared key heads, causal with a prefix that all
           see, capped scores, a bias by distance (of positions, or of voxels in space)

``run`` computes a pass with elementary torch operations in float32 where ``own`` is false,
and through the package's entry points where it is true.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
SMALLEST = 2.0 ** -126  # least scale of a block: a block of zeros gets it
BLOCK = 128
EPS = 1e-6


def listed():
    return [
        # one new token of a decoder: the norm before its products; latency is all
        {"name": "norm_token_bf16_c1024", "kind": "norm", "n": 1, "c": 1024, "dtype": "bf16", "res": True, "bits8": True,
         "pad": 0},
        # the voxels of a coarse level of two frames, at the width of the networks' last stage
        {"name": "norm_voxels_f16_c256", "kind": "norm", "n": 11_003, "c": 256, "dtype": "f16", "res": True, "bits8": True,
         "pad": 0},
        # float32 rows of an odd width inside wider rows (a slice of a fused product), kept in float32
        {"name": "norm_slice_f32_c1000", "kind": "norm", "n": 4099, "c": 1000, "dtype": "f32", "res": False,
         "bits8": False, "pad": 536},
        # a long prompt, or a batch of whole scenes, at a wide model
        {"name": "norm_large_bf16_c4096", "kind": "norm", "n": 65_536, "c": 4096, "dtype": "bf16", "res": True,
         "bits8": True, "pad": 0},
        # one new token: reading the weights is all
        {"name": "linear_token_bf16", "kind": "linear", "m": 1, "n": 4096, "k": 1024, "dtype": "bf16", "relu": False},
        # a batch of new tokens, an odd number of outputs
        {"name": "linear_tokens_f32_odd", "kind": "linear", "m": 33, "n": 1001, "k": 4096, "dtype": "f32", "relu": False},
        # query, key and value features of the voxels of a coarse level
        {"name": "linear_voxels_f16", "kind": "linear", "m": 11_003, "n": 768, "k": 256, "dtype": "f16", "relu": False},
        # the wide product of a long prompt
        {"name": "linear_large_bf16", "kind": "linear", "m": 16_384, "n": 8192, "k": 4096, "dtype": "bf16", "relu": True},
        # one new token against a short cache, capped scores
        {"name": "attend_token_bf16", "kind": "attend", "docs": 1, "q_max": 1, "k_max": 2049, "hq": 8, "hkv": 2, "d": 64,
         "dtype": "bf16", "causal": True, "prefix": False, "cap": 30.0, "bias": "none"},
        # a batch of documents, one new token each, caches of very different lengths
        {"name": "attend_cache_bf16", "kind": "attend", "docs": 48, "q_max": 1, "k_max": 8192, "hq": 32, "hkv": 8,
         "d": 128, "dtype": "bf16", "causal": True, "prefix": False, "cap": 0.0, "bias": "position"},
        # the voxels of two frames at a coarse level: every voxel sees its frame, nearer ones count more
        {"name": "attend_voxels_f16", "kind": "attend", "docs": 2, "q_max": 0, "k_max": 5803, "hq": 8, "hkv": 8, "d": 32,
         "dtype": "f16", "causal": False, "prefix": False, "cap": 0.0, "bias": "voxel"},
        # whole documents: a scene's tokens as the prefix, text after it; capped scores
        {"name": "attend_prefix_bf16", "kind": "attend", "docs": 3, "q_max": 0, "k_max": 8192, "hq": 16, "hkv": 4,
         "d": 128, "dtype": "bf16", "causal": True, "prefix": True, "cap": 50.0, "bias": "none"},
    ]


def draw(rng):
    def between(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    kind = rng.choice(["norm", "linear", "attend", "attend"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    if kind == "norm":
        bits8 = rng.random() < 0.7
        c = 16 * between(1, 512) if bits8 else between(1, 8192)
        n = between(1, max(2, min(65_536, 190_000_000 // c)))
        return {"kind": kind, "n": n, "c": c, "dtype": dtype, "res": rng.random() < 0.7, "bits8": bits8,
                "pad": rng.choice([0, 0, 16, 104])}
    if kind == "linear":
        m, n, k = between(1, 16_384), between(1, 8192), 16 * between(1, 512)
        while m * n * k > 400_000_000_000:
            m = max(1, m // 2)
        return {"kind": kind, "m": m, "n": n, "k": k, "dtype": dtype, "relu": rng.random() < 0.3}
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 1, 2, 3, 4, 8])
    d = rng.choice([16, 32, 64, 64, 80, 96, 128, 128, 256])
    whole = rng.random() < 0.5
    bias = rng.choice(["none", "none", "position", "voxel"])
    causal = rng.random() < 0.6
    case = {"kind": kind, "docs": between(1, 8 if whole else 64), "q_max": 0 if whole else rng.choice([1, 1, 1, 2, 5, 77, 300]),
            "k_max": between(1, 6000), "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "causal": causal,
            "prefix": causal and rng.random() < 0.5, "cap": rng.choice([0.0, 0.0, 20.0, 50.0]), "bias": bias}
    # at most a sixteenth of the largest listed case's pairs in float32, whose products cost more
    while case["docs"] * hq * (case["q_max"] or case["k_max"]) * case["k_max"] * d > (1 << 38 if dtype != "f32" else 1 << 35):
        case["k_max"] = max(1, case["k_max"] // 2)
        case["docs"] = max(1, case["docs"] * 3 // 4)
    return case


# ----------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------

def _lengths(case):
    """(queries, keys, prefix) of each document: the first is the longest, the others spread
    below it; a batch of caches holds an empty one."""
    docs, most, few = case["docs"], case["k_max"], case["q_max"]
    k = [most if i == 0 else max(1, most * ((i * 37 + 11) % 89 + 4) // 93) for i in range(docs)]
    if few and docs > 3:
        k[2] = 0
    # an empty cache still has its queries: they see nothing
    q = list(k) if not few else [few if n == 0 else min(n, few - i % 2 if few > 1 else 1) for i, n in enumerate(k)]
    p = [n // 3 if case["prefix"] else 0 for n in k]
    return q, k, p


def _gen(seed):
    return torch.Generator(DEV).manual_seed(9_000_011 + seed)


def _quantize(x, cols):
    """x as e4m3 and float32 scales, one scale for each block of 128 columns and of `cols` rows."""
    n, c = x.shape
    kb, nb = -(-c // BLOCK), -(-n // cols)
    wide = torch.zeros((nb * cols, kb * BLOCK), dtype=torch.float32, device=x.device)
    wide[:n, :c] = x
    wide = wide.view(nb, cols, kb, BLOCK)
    scale = (wide.abs().amax((1, 3)) / E4M3_MAX).clamp(min=SMALLEST)
    q = (wide / scale[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).view(nb * cols, kb * BLOCK)[:n, :c]
    return q.contiguous().to(E4M3), scale


def prepare(case, seed):
    g, s, kind = _gen(seed), {"case": case}, case["kind"]

    def normal(*shape):
        return torch.randn(shape, device=DEV, generator=g)

    if kind == "norm":
        n, c, dt = case["n"], case["c"], DT[case["dtype"]]
        # residual streams: rows of different size, a few channels that stand out
        big = 1.0 + 20.0 * (torch.rand(c + case["pad"], device=DEV, generator=g) < 0.01)
        rows = torch.exp(0.5 * normal(n, 1))
        s["x"] = (normal(n, c + case["pad"]) * rows * big).to(dt)[:, :c]
        s["gamma"] = (1.0 + 0.1 * normal(c)).to(dt)
        s["res"] = (normal(n, c) * rows).to(dt) if case["res"] else None
        return s
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s["xq"], s["xs"] = _quantize(normal(m, k), 1)
        s["wq"], s["ws"] = _quantize(normal(n, k) / math.sqrt(k), BLOCK)
        return s
    ql, kl, pl = _lengths(case)
    hq, hkv, d, dt = case["hq"], case["hkv"], case["d"], DT[case["dtype"]]
    s["max_q"], s["max_k"] = max(ql), max(kl)
    starts = lambda v: torch.tensor(np.concatenate([[0], np.cumsum(v)]), dtype=torch.int32, device=DEV)  # noqa: E731
    s["q_start"] = starts(ql)
    if case["q_max"] == 0:
        # one fused product holds the queries, keys and values of a row
        rows = normal(sum(kl), (hq + 2 * hkv) * d).to(dt)
        s["q"], s["k"], s["v"] = (t.unflatten(1, (-1, d)) for t in rows.split([hq * d, hkv * d, hkv * d], 1))
        s["k_start"], s["k_len"] = s["q_start"], None
    else:
        # a cache: room for k_max keys of each document
        s["q"] = normal(sum(ql), hq, d).to(dt)
        s["k"], s["v"] = (normal(case["docs"] * case["k_max"], hkv, d).to(dt) for _ in range(2))
        s["k_start"] = starts([case["k_max"]] * case["docs"])
        s["k_len"] = torch.tensor(kl, dtype=torch.int32, device=DEV)
    s["prefix"] = torch.tensor(pl, dtype=torch.int32, device=DEV) if case["prefix"] else None
    s["slopes"] = s["q_pos"] = s["k_pos"] = None
    if case["bias"] != "none":
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device=DEV) / hq)
    if case["bias"] == "voxel":
        # voxels of the third downsampling level of 100 m frames: multiples of 8
        def voxels(n):
            return 8 * torch.randint(-125, 125, (n, 4), device=DEV, generator=g, dtype=torch.int32)

        s["k_pos"] = voxels(len(s["k"]))
        s["q_pos"] = s["k_pos"] if case["q_max"] == 0 else voxels(len(s["q"]))
        s["slopes"] = s["slopes"] / 8
    return s


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------

def run(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        if own:
            from paper_2401_06145_amd import binding as B

            y, scale, total = B.rms_norm(s["x"], s["gamma"], residual=s["res"], eps=EPS, bits8=case["bits8"])
        else:
            y, scale, total = _norm(s, case)
        return {"y": y, "scale": scale, "sum": total}
    if kind == "linear":
        if own:
            from paper_2401_06145_amd import binding as B

            return B.scaled_linear(s["xq"], s["xs"], s["wq"], s["ws"], DT[case["dtype"]], relu=case["relu"])
        return _linear(s, case)
    if own:
        from paper_2401_06145_amd import binding as B

        return B.attention(s["q"], s["k"], s["v"], s["q_start"], s["k_start"], s["max_q"], s["max_k"], k_len=s["k_len"],
                           prefix=s["prefix"], causal=case["causal"], cap=case["cap"], slopes=s["slopes"],
                           q_pos=s["q_pos"], k_pos=s["k_pos"])
    return _attend(s, case)


def _norm(s, case):
    x = s["x"].float()
    total = None
    if s["res"] is not None:
        x = x + s["res"].float()
        total = x.to(s["x"].dtype)
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * s["gamma"].float()
    if not case["bits8"]:
        return y.to(s["x"].dtype), None, total
    q, scale = _quantize(y, 1)
    return q, scale, total


def _spread(scale, rows, shape):
    """Block scales as one factor for each element."""
    return scale.repeat_interleave(rows, 0)[:shape[0]].repeat_interleave(BLOCK, 1)[:, :shape[1]]


def _linear(s, case):
    x = s["xq"].float() * _spread(s["xs"], 1, s["xq"].shape)
    w = s["wq"].float() * _spread(s["ws"], BLOCK, s["wq"].shape)
    y = x @ w.t().contiguous()
    if case["relu"]:
        y = y.clamp(min=0.0)
    return y.to(DT[case["dtype"]])


def _attend(s, case):
    """The documents as a padded batch."""
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    hq, hkv, d, docs = case["hq"], case["hkv"], case["d"], case["docs"]
    mq, mk, g = s["max_q"], s["max_k"], hq // hkv
    qs, ks = s["q_start"].long(), s["k_start"].long()
    ql = qs[1:] - qs[:-1]
    kl = ks[1:] - ks[:-1] if s["k_len"] is None else s["k_len"].long()
    at_q, at_k = torch.arange(mq, device=DEV), torch.arange(mk, device=DEV)
    rows_q = (qs[:-1, None] + at_q).clamp(max=len(q) - 1)
    rows_k = (ks[:-1, None] + at_k).clamp(max=len(k) - 1)
    there = at_k < kl[:, None]  # [docs, mk]
    qp = q[rows_q].view(docs, mq, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(docs, hkv, g * mq, d)
    kp = k[rows_k].permute(0, 2, 3, 1).contiguous()
    vp = (v[rows_k] * there[:, :, None, None]).permute(0, 2, 1, 3).contiguous()
    score = (qp @ kp).view(docs, hkv, g, mq, mk) / math.sqrt(d)
    if case["cap"] > 0:
        score = case["cap"] * torch.tanh(score / case["cap"])
    # a query's place among its document's keys: the last query is the last key
    place = at_q + (kl - ql)[:, None]  # [docs, mq]
    if case["bias"] == "position":
        far = (place[:, :, None] - at_k).abs().float()
    elif case["bias"] == "voxel":
        far = 0.0
        for axis in (1, 2, 3):
            far = far + (s["q_pos"][:, axis].float()[rows_q][:, :, None] - s["k_pos"][:, axis].float()[rows_k][:, None]).square()
        far = far.sqrt()
    if case["bias"] != "none":
        score = score - s["slopes"].view(1, hkv, g, 1, 1) * far[:, None, None]
    seen = there[:, None].expand(docs, mq, mk)
    if case["causal"]:
        most = place + 1
        if s["prefix"] is not None:
            most = torch.maximum(most, s["prefix"].long()[:, None])
        seen = seen & (at_k < most[:, :, None])
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    del score
    total = p.sum(-1)
    out = (p.view(docs, hkv, g * mq, mk) @ vp).view(docs, hkv, g, mq, d) / torch.where(total == 0, 1.0, total)[..., None]
    out = out.permute(0, 3, 1, 2, 4).reshape(docs, mq, hq, d)
    row = torch.arange(len(q), device=DEV)
    doc = torch.searchsorted(qs, row, right=True) - 1
    return out[doc, row - qs[doc]].to(s["q"].dtype)


# ----------------------------------------------------------------------------
# The same in 64 bits
# ----------------------------------------------------------------------------

def _round_e4m3(v):
    """The nearest number with 3 bits after the point and exponents from -6, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "norm":
        x = s["x"].double()
        if s["res"] is not None:
            x = x + s["res"].double()
        total = x if s["res"] is not None else None
        y = x * s["gamma"].double() / ((x ** 2).sum(1, keepdim=True) / case["c"] + EPS).sqrt()
        if not case["bits8"]:
            return {"y": y, "scale": None, "sum": total}
        scales = []
        for b in range(0, case["c"], BLOCK):
            part = y[:, b:b + BLOCK]
            scales.append((part.abs().max(1).values / E4M3_MAX).clamp(min=SMALLEST))
            y[:, b:b + BLOCK] = _round_e4m3(part / scales[-1][:, None])
        return {"y": y, "scale": torch.stack(scales, 1), "sum": total}
    if kind == "linear":
        y = torch.zeros((case["m"], case["n"]), dtype=torch.float64, device=DEV)
        for b in range(0, case["k"], BLOCK):
            x = s["xq"][:, b:b + BLOCK].double() * s["xs"][:, b // BLOCK, None].double()
            w = s["wq"][:, b:b + BLOCK].double()
            for r in range(0, case["n"], BLOCK):
                w[r:r + BLOCK] *= s["ws"][r // BLOCK, b // BLOCK].double()
            y += x @ w.t().contiguous()
        return y.relu() if case["relu"] else y
    ql, kl, pl = _lengths(case)
    if sum(a * b for a, b in zip(ql, kl)) * case["hq"] * case["d"] > 6e12:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    starts_q, starts_k = s["q_start"].tolist(), s["k_start"].tolist()
    for i, (nq, nk, pre) in enumerate(zip(ql, kl, pl)):
        if nq == 0 or nk == 0:
            continue
        a, b = slice(starts_q[i], starts_q[i] + nq), slice(starts_k[i], starts_k[i] + nk)
        ahead = torch.arange(nq, device=DEV)[:, None] + (nk - nq) - torch.arange(nk, device=DEV)[None]
        hidden = (ahead < 0) & (torch.arange(nk, device=DEV)[None] >= pre) if case["causal"] else torch.zeros_like(ahead, dtype=torch.bool)
        if case["bias"] == "position":
            far = ahead.abs().double()
        elif case["bias"] == "voxel":
            far = (s["q_pos"][a, None, 1:].double() - s["k_pos"][None, b, 1:].double()).norm(dim=2)
        for h in range(case["hq"]):
            kv = h * case["hkv"] // case["hq"]
            t = s["q"][a, h].double() @ s["k"][b, kv].double().t().contiguous() * case["d"] ** -0.5
            if case["cap"] > 0:
                t = torch.tanh(t / case["cap"]) * case["cap"]
            if case["bias"] != "none":
                t = t - s["slopes"][h].double() * far
            t = torch.softmax(t.masked_fill(hidden, -math.inf), 1)
            # a row that sees no key gives zeros
            out[a, h] = torch.where(hidden.all(1, keepdim=True), 0.0, t) @ s["v"][b, kv].double()
    return out


# ----------------------------------------------------------------------------
# What a pass cannot do without
# ----------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    e = 4 if case["dtype"] == "f32" else 2
    if kind == "norm":
        n, c = case["n"], case["c"]
        y = n * c + 4 * n * -(-c // BLOCK) if case["bits8"] else e * n * c
        return {"bytes": float(e * n * c * (3 if case["res"] else 1) + e * c + y), "flops": 0}
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        kb = -(-k // BLOCK)
        return {"bytes": float((m + n) * k + e * m * n + 4 * kb * (m + -(-n // BLOCK))), "flops": 2.0 * m * n * k}
    ql, kl, pl = _lengths(case)
    pairs, d = 0, case["d"]
    for nq, nk, pre in zip(ql, kl, pl):
        most = np.arange(nq, dtype=np.int64) + (nk - nq) + 1 if case["causal"] else np.full(nq, nk, dtype=np.int64)
        pairs += int(np.clip(np.maximum(most, pre), 0, nk).sum())
    byts = 2.0 * sum(ql) * case["hq"] * d * e + 2.0 * sum(kl) * case["hkv"] * d * e
    if case["bias"] == "voxel":
        byts += 16.0 * (sum(kl) + (sum(ql) if case["q_max"] else 0))
    return {"bytes": byts, "flops": 4.0 * pairs * case["hq"] * d}
