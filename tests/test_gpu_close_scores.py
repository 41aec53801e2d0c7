"""Attention where many scores are large and close to each other: every part of a row (tiles, waves, ranges of keys) has
a maximum of its own, and the parts' weights go by small differences of large numbers."""
from __future__ import annotations

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests import cache_ref as cref
from tests import transformer_ref as ref
from tests.cache_ref import Cached, check_attention
from tests.gpu_helpers import DEV, say

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
D, SCALE = 64, 0.125

# Of a score's two products one is the same for all keys, 448 times q[0], and one a multiple of 1/8 below 2; each is a
# number of every type (keys of 8 bits have a scale of 1), and the sum one of float32: scores are exact.
FIRST = {150: 43 / 128, 200: 29 / 64, 1000: 2.25, 12_500: 28.0, 125_000: 280.0, 500_000: 1120.0}


def documents(ql, kl, heads, kv, dtype, bits8, size, sign, order):
    g = torch.Generator(DEV).manual_seed(size % 997)
    k = torch.zeros((sum(kl), kv, D), device=DEV)
    k[..., 0] = 448.0 * sign
    for t, n in enumerate(kl):
        at = torch.arange(n, device=DEV)
        steps = {"rising": at * 16 // n, "falling": (n - 1 - at) * 16 // n,
                 "mixed": torch.randint(0, 16, (n,), device=DEV, generator=g)}[order]
        k[sum(kl[:t]):sum(kl[:t + 1]), :, D // 2 + 9] = (steps / 8.0)[:, None]
    b = Cached(ql, kl, heads, kv, D, dtype, bits8, 32, seed=size % 991,
               like=(k, torch.randn((sum(kl), kv, D), device=DEV, generator=g)))
    b.q[:] = 0.0
    b.q[..., 0] = FIRST[size] / SCALE
    b.q[..., D // 2 + 9] = 1.0 / SCALE
    return b


# one token and few queries; many queries; lengths that are split into ranges and not
SHAPES = [([1], [300], 1, 1), ([3, 1], [5000, 90], 8, 2), ([150], [400], 4, 2), ([150], [6000], 2, 1)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("size", FIRST)
def test_over_pages(size, bits8, dtype):
    for shape in SHAPES:
        for sign in (1, -1):
            for order in ("rising", "falling", "mixed"):
                say(f"scores of {sign * size}, {order}, over pages {shape}, 8 bits {bits8} {dtype}")
                b = documents(*shape, dtype, bits8, size, sign, order)
                for kw in (dict(), dict(slopes=torch.zeros(shape[2], device=DEV))):
                    check_attention(b.run(scale=SCALE, causal=False, **kw), *b.want(scale=SCALE, causal=False, **kw),
                                    f"{sign * size} {order} {shape}")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("size", FIRST)
def test_over_packed_keys(size, dtype):
    for shape in SHAPES:
        for sign in (1, -1):
            for order in ("rising", "falling", "mixed"):
                say(f"scores of {sign * size}, {order}, over packed keys {shape} {dtype}")
                b = documents(*shape, dtype, False, size, sign, order)
                ql, kl = shape[:2]
                got = B.attention(b.q, b.k.to(dtype), b.v.to(dtype), b.q_start, cref.starts(kl), max(ql), max(kl), scale=SCALE)
                check_attention(got, *b.want(scale=SCALE, causal=False), f"{sign * size} {order} {shape}")


def test_steep_slopes_over_packed_keys():
    """Biases far beyond the exponentials' range, of either sign."""
    say("steep slopes over packed keys")
    for ql, kl in (([3, 1], [700, 90]), ([150, 70], [200, 3000])):
        for dtype in (F32, F16, BF16):
            b = Cached(ql, kl, 8, 2, D, dtype, seed=13)
            slopes = torch.tensor([0.0, 1e-3, 1.0, -1e-2, 1e9, 1e12, 1e20, 1e37], device=DEV)
            got = B.attention(b.q, b.k.to(dtype), b.v.to(dtype), b.q_start, cref.starts(kl), max(ql), max(kl), causal=True,
                              slopes=slopes)
            check_attention(got, *b.want(slopes=slopes), f"{ql} of {kl} {dtype}")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("bits8", [False, True])
def test_rows_do_not_go_by_others(bits8, dtype):
    """A row with large scores beside one with small ones: the latter's bits are what they were."""
    say(f"one row of large scores, 8 bits {bits8} {dtype}")
    for ql, kl in (([4, 2], [700, 90]), ([150, 70], [400, 900])):
        b = Cached(ql, kl, 4, 2, D, dtype, bits8, 16, seed=17)
        clean = b.run()
        b.q[1, 2] *= 300.0
        got = b.run()
        got[1, 2] = clean[1, 2]
        assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("source", ["pages", "pages of 8 bits", "packed"])
@pytest.mark.parametrize("slopes", [[-0.25, -0.25], [0.25, -0.25]])
def test_far_keys_of_negative_slopes(slopes, source, dtype):
    """Far keys with large biases: what their products add is small beside those, and must not be lost step by step.
    Biases are multiples of 128 from 2^20 on in units of the products, where float32's step is 1/8; every second key has 96
    products of 2^-8, together 3 steps, of which 16 are half of one.  Bias, product and sum are float32 numbers."""
    say(f"slopes {slopes}, {source} {dtype}")
    n, nq, d = 66_000, 150, 128
    k = torch.zeros((n, 1, d), device=DEV)
    k[::2, :, :96] = 2.0 ** -5
    k[..., 127] = 448 * 2.0 ** -9  # (rows of 8 bits have a scale of 2^-9)
    g = torch.Generator(DEV).manual_seed(18)
    b = Cached([nq], [n], 2, 1, d, dtype, source == "pages of 8 bits", 32, seed=18,
               like=(k, torch.randn((n, 1, d), device=DEV, generator=g)))
    b.q[:] = 0.0
    b.q[..., :96] = 2.0 ** -3
    kw = dict(scale=2.0 ** -6, slopes=torch.tensor(slopes, device=DEV))
    if source == "packed":
        got = B.attention(b.q, b.k.to(dtype), b.v.to(dtype), b.q_start, cref.starts([n]), nq, n, causal=True, **kw)
    else:
        got = b.run(**kw)
    check_attention(got, *b.want(**kw), source)


def test_queries_before_the_first_key():
    """More queries than keys: the first stand before all keys, and see a prefix of them from afar.

    A score of a bias of up to 2 x 700 is rounded to float32 where the bias is added, by at most 1400 x 2^-24 (half a step
    relative to its size), which is a factor of as much of its exponential: of each of a row's sum of values and
    its sum of exponentials, so of their quotient twice that, 1.7e-4, beside what the bound counts anyway (products, and
    distances of some hundred)."""
    say("queries before the first key, with slopes")
    for dtype in (F32, F16, BF16):
        for bits8 in (False, True):
            b = Cached([700, 150], [90, 300], 4, 2, D, dtype, bits8, 16, seed=19)
            slopes = torch.tensor([0.5, -0.5, 0.01, 2.0], device=DEV)
            for kw in (dict(prefix=[40, 5]), dict(causal=False)):
                got, (want, mag) = b.run(slopes=slopes, **kw), b.want(slopes=slopes, **kw)
                u = ref.UNIT[dtype]
                bound = mag * (2 * u + 4e-5 + 2 * 1400 * 2.0 ** -24) + want.abs() * u + 2 * ref.TINY[dtype]
                off = (got.double() - want).abs()
                assert bool((off <= bound).all()), f"{kw} {dtype}: off by {float((off / bound).max()):.2f} of the bound"
