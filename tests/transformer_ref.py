"""The transformer operators in 64 bits, written out plainly, and the bounds their results
are held to (derived from the formats, not from runs)."""
from __future__ import annotations

import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# least step of a type's subnormal numbers, halved
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def rms_norm(x, gamma, residual=None, eps=1e-6):
    s = x.double() + (0 if residual is None else residual.double())
    return s / torch.sqrt((s * s).mean(1, keepdim=True) + eps) * gamma.double(), s


def block_top(y):
    """Largest magnitude of each 128 columns."""
    n, c = y.shape
    wide = torch.zeros((n, -(-c // 128) * 128), dtype=y.dtype, device=y.device)
    wide[:, :c] = y.abs()
    return wide.view(n, -1, 128).amax(2)


def spread(scale, c):
    return scale.double().repeat_interleave(128, 1)[:, :c]


def check_rows(got, want, c, what):
    """A row value in the rows' type: one rounding, and float32 arithmetic (a sum of c squares in
    order of at most c / 16 terms a lane, a root, a division and two products)."""
    slack = (c / 16 + 16) * 2.0 ** -24
    bound = want.abs() * (UNIT[got.dtype] + slack) + TINY[got.dtype]
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"{what}: off by {float((off / bound).max()):.2f} of the bound"


def check_bits8(q, scale, want, what):
    """Scales within float32 arithmetic; values within half a step of e4m3 at their size."""
    c = want.shape[1]
    slack = (c / 16 + 16) * 2.0 ** -24
    top = (block_top(want) / 448.0).clamp(min=2.0 ** -126)
    assert bool(((scale.double() - top).abs() <= top * (slack + 2.0 ** -23)).all()), f"{what}: scales"
    step = torch.maximum(want.abs() * 2.0 ** -4, spread(scale, c) * 2.0 ** -10)
    off = (q.float().double() * spread(scale, c) - want).abs()
    bound = step * (1 + 2.0 ** -10) + want.abs() * slack
    assert bool((off <= bound).all()), f"{what}: off by {float((off / bound).max()):.3f} of half a step"


def scaled_linear(xq, xs, wq, ws, relu=False):
    """(result, sum of magnitudes) of the product."""
    k = xq.shape[1]
    x = xq.float().double() * spread(xs, k)
    w = wq.float().double() * spread(ws, k).repeat_interleave(128, 0)[:wq.shape[0]]
    y = x @ w.t().contiguous()
    return (y.relu() if relu else y), x.abs() @ w.abs().t().contiguous()


def check_linear(got, want, mag, k, what):
    """Sums of float32 in any order: k terms, at 2^-24 of the magnitudes' sum each; one rounding."""
    bound = mag * ((min(k, 128) + k / 128 + 4) * 2.0 ** -24) + want.abs() * UNIT[got.dtype] + TINY[got.dtype]
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"{what}: off by {float((off / bound).max()):.2f} of the bound"


def attention(q, k, v, q_lens, k_lens, k_starts=None, prefix=None, causal=False, scale=None, cap=0.0, slopes=None,
              q_pos=None, k_pos=None):
    """(result, sums of p |v|) over documents given by Python lists."""
    heads, d = q.shape[1], q.shape[2]
    group = heads // k.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    mag = torch.zeros_like(out)
    scale = 1 / math.sqrt(d) if scale is None else scale
    q0, at = 0, 0
    for t, (nq, nk) in enumerate(zip(q_lens, k_lens)):
        k0 = at if k_starts is None else k_starts[t]
        at += nk
        if nq and nk:
            i = torch.arange(nq, device=q.device)[:, None] + nk - nq
            j = torch.arange(nk, device=q.device)[None]
            see = torch.ones((nq, nk), dtype=torch.bool, device=q.device)
            if causal:
                see = (j <= i) | (j < (0 if prefix is None else prefix[t]))
            for h in range(heads):
                # as a CPU product: hidden rows may hold anything, and 0 * NaN must not spread
                kk, vv = k[k0:k0 + nk, h // group].double(), v[k0:k0 + nk, h // group].double()
                s = q[q0:q0 + nq, h].double() @ kk.t().contiguous() * scale
                if cap > 0:
                    s = cap * torch.tanh(s / cap)
                if slopes is not None:
                    if q_pos is not None:
                        far = (q_pos[q0:q0 + nq, None, 1:].double() - k_pos[None, k0:k0 + nk, 1:].double()).square().sum(2).sqrt()
                    else:
                        far = (i - j).abs().double()
                    s = s - slopes[h].double() * far
                s = torch.where(see, s, -math.inf)
                top = s.amax(1, keepdim=True)
                p = torch.where(see, torch.exp(s - torch.where(top == -math.inf, 0.0, top)), 0.0)
                p = p / torch.where(top == -math.inf, 1.0, p.sum(1, keepdim=True))
                out[q0:q0 + nq, h] = p @ vv
                mag[q0:q0 + nq, h] = p @ vv.abs()
        q0 += nq
    return out, mag


def check_attention(got, want, mag, what):
    """Exponentials rounded to the rows' type once (and their sum, which is not, so twice in the
    quotient at most); scores in float32: products of up to 256 terms, a tanh of 2^-23 times the
    cap, a distance of up to some hundred, together within 4e-5; one rounding of the result."""
    u = UNIT[got.dtype]
    bound = mag * (2 * u + 4e-5) + want.abs() * u + TINY[got.dtype]
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"{what}: off by {float((off / bound).max()):.2f} of the bound"
