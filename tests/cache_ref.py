"""The operators of a paged cache in 64 bits, written out plainly, and the bounds their results are
held to (derived from the formats, not from runs)."""
from __future__ import annotations

import math

import torch

from paper_2401_06145_amd import binding as B
from tests import transformer_ref as ref
from tests.gpu_helpers import DEV

E4M3_HALF = 2.0 ** -4  # half a step, relative to the value


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def starts(lens):
    return ints([sum(lens[:i]) for i in range(len(lens) + 1)])


def rotate(x, pos, freq, gamma=None, eps=1e-6, interleaved=False, gain=1.0):
    """(result, sum of magnitudes) of heads x [n][h][d]; pos [n] or [n][4]."""
    rot = 2 * len(freq)
    y = x.double()
    if gamma is not None:
        y = y / torch.sqrt((y * y).mean(2, keepdim=True) + eps) * gamma.double()
    out, mag = y.clone(), y.abs()
    for j in range(len(freq)):
        p = (pos if pos.dim() == 1 else pos[:, 1 + j % 3]).double()
        c, s = (gain * torch.cos(p * freq[j]))[:, None], (gain * torch.sin(p * freq[j]))[:, None]
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., a] * s + y[..., b] * c
        both = abs(gain) * (y[..., a].abs() + y[..., b].abs())
        mag[..., a], mag[..., b] = both, both
    return out, mag


def check_rotated(got, want, mag, what):
    """A sum of up to 256 squares in float32, a root, a quotient and two products; an angle's fraction of a
    turn in float32 (2^-26 turns, and as much again from the float64 product), cosine and sine
    within four roundings, two products and a sum: together d + 24 roundings at most; one of
    the result."""
    slack = (want.shape[2] + 24) * 2.0 ** -24
    bound = mag * slack + want.abs() * ref.UNIT[got.dtype] + ref.TINY[got.dtype]
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"{what}: off by {float((off / bound).max()):.2f} of the bound"


def check_rows8(q, scale, x, what):
    """Scales: a maximum and one quotient.  Values: within half a step of x / scale at its size (subnormal
    steps are 2^-9), by a quotient in float32."""
    want = (x.double().abs().amax(-1) / 448.0).clamp(min=2.0 ** -126)
    assert bool(((scale.double() - want).abs() <= want * 2.0 ** -23).all()), f"{what}: scales"
    by = scale.double()[..., None]
    off = (q.float().double() * by - x.double()).abs()
    bound = torch.maximum(x.double().abs() * E4M3_HALF, by * 2.0 ** -10) * (1 + 2.0 ** -10)
    assert bool((off <= bound).all()), f"{what}: off by {float((off / bound).max()):.3f} of half a step"


class Cached:
    """Documents with the given keys in pages that are given out in a shuffled order.  What no call may
    use (free pages, rows behind a document's last) holds NaN."""

    def __init__(self, q_lens, k_lens, heads, kv_heads, d, dtype, bits8=False, page=16, seed=0, spread=1.0, spare=3,
                 wide=1, like=None):
        g = torch.Generator(DEV).manual_seed(seed)
        self.q_lens, self.k_lens, self.page, self.bits8, self.dtype = q_lens, k_lens, page, bits8, dtype
        self.heads, self.kv_heads, self.d = heads, kv_heads, d

        def normal(*shape):
            return torch.randn(shape, device=DEV, generator=g)

        self.q = (normal(sum(q_lens), heads, d) * spread).to(dtype)
        need = [-(-n // page) for n in k_lens]
        pages = sum(need) + spare
        order = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)
        self.table = torch.full((len(k_lens), max(need, default=0) + wide), -7, dtype=torch.int32, device=DEV)
        at = 0
        for t, m in enumerate(need):
            self.table[t, :m] = order[at:at + m]
            at += m
        k, v = (normal(sum(k_lens), kv_heads, d) for _ in range(2)) if like is None else like
        self.cache = B.Pages.make(pages, page, kv_heads, d, dtype, bits8, DEV)
        for name in ("k", "v"):
            getattr(self.cache, name).view(torch.uint8).fill_(0x7f if bits8 else 0xff)  # NaN in every type
            if bits8:
                getattr(self.cache, name + "_scale").fill_(math.nan)
        self.k, self.v = (torch.cat([self.put(name, t, x[sum(k_lens[:t]):sum(k_lens[:t + 1])]) for t in range(len(k_lens))])
                          if len(k_lens) else x for name, x in (("k", k), ("v", v)))
        self.q_start, self.k_len = starts(q_lens), ints(k_lens)

    def put(self, name, t, rows):
        """Document t's rows [n][kv_heads][d] into its pages by torch; the values that the pages stand for."""
        place = torch.arange(len(rows), device=DEV)
        at = self.table[t].long()[place // self.page]
        store = getattr(self.cache, name)
        if not self.bits8:
            store[at, :, place % self.page] = rows.to(self.dtype)
            return rows.to(self.dtype).double()
        x = rows.to(self.dtype).float()
        scale = (x.abs().amax(2) / 448.0).clamp(min=2.0 ** -126)
        q = (x / scale[..., None]).clamp(-448.0, 448.0).to(B.E4M3)
        store.view(torch.uint8)[at, :, place % self.page] = q.view(torch.uint8)
        getattr(self.cache, name + "_scale")[at, :, place % self.page] = scale
        return q.float().double() * scale.double()[..., None]

    def run(self, **kw):
        a = dict(q=self.q, cache=self.cache, q_start=self.q_start, k_len=self.k_len, table=self.table,
                 max_q=max(self.q_lens, default=0), max_k=max(self.k_lens, default=0))
        if kw.get("prefix") is not None:
            kw["prefix"] = ints(kw["prefix"])
        return B.cached_attention(**{**a, **kw})

    def want(self, **kw):
        kw.setdefault("causal", True)
        return ref.attention(self.q, self.k, self.v, self.q_lens, self.k_lens, **kw)


def check_attention(got, want, mag, what):
    """As over packed keys: exponentials (8-bit pages: times a scale's mantissa) rounded to the rows'
    type once; float16 rows of 8-bit pages may be rounded to float16's subnormals."""
    u = ref.UNIT[got.dtype]
    bound = mag * (2 * u + 4e-5) + want.abs() * u + 2 * ref.TINY[got.dtype]
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"{what}: off by {float((off / bound).max()):.2f} of the bound"
