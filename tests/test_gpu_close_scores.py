"""Attention where many scores are large and close to each other: every part of a row (tiles, waves, ranges of keys) has
a maximum of its own, and the parts' weights go by small differences of large numbers."""
from __future__ import annotations

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests import cache_ref as cref
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
