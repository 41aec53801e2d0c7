"""The transformer operators' torch binding on rows and heads whose strides do not count, or that lie
oddly: a single row of an odd array, scales of more columns than blocks."""
from __future__ import annotations

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests import transformer_ref as ref
from tests.gpu_helpers import DEV, say
from tests.test_gpu_attention import ints
from tests.test_gpu_scaled_linear import bits8, scales

pytestmark = pytest.mark.gpu


def test_a_single_row_of_an_odd_array():
    """Row 2 of rows 1016 bytes apart begins at a multiple of 16; the distance to the next is nobody's concern."""
    say("operators on a single row of an odd array")
    n, k = 200, 960
    x, w = bits8(3, k, 1, pad=56)[2:3], bits8(n, k, 2)
    xs, ws = scales(1, k, 3), scales(2, k, 4)
    assert x.stride(0) == 1016
    want, mag = ref.scaled_linear(x, xs, w, ws)
    ref.check_linear(B.scaled_linear(x, xs, w, ws, torch.float32), want, mag, k, "one row")
    y = torch.empty((1, n), device=DEV)
    B.spconv_scaled_linear(x, xs, w, ws, y)
    ref.check_linear(y, want, mag, k, "one row, given output")
    one = bits8(3, k, 5, pad=56)[2:3]
    want, mag = ref.scaled_linear(w, scales(n, k, 6), one, scales(1, k, 7))
    ref.check_linear(B.scaled_linear(w, scales(n, k, 6), one, scales(1, k, 7), torch.float32), want, mag, k, "one output")


def test_a_single_row_or_head_of_attention():
    say("attention on a single row and a single head of odd arrays")
    g = torch.Generator(DEV).manual_seed(8)
    d, n = 64, 40
    wide = torch.randn((3, 2 * d + 4), device=DEV, generator=g).to(torch.float16)
    q = wide.as_strided((1, 2, d), (2 * d + 4, d, 1), 2 * (2 * d + 4))
    k, v = (torch.randn((n, 2, d), device=DEV, generator=g).to(torch.float16) for _ in range(2))
    assert q.stride(0) * 2 % 16 != 0
    want, mag = ref.attention(q, k, v, [1], [n])
    ref.check_attention(B.attention(q, k, v, ints([0, 1]), ints([0, n]), 1, n), want, mag, "one row")
    q1, k1, v1 = (t[:, :1].contiguous().as_strided((len(t), 1, d), (d, 3, 1)) for t in (torch.randn((n, 1, d), device=DEV,
                  generator=g).to(torch.float16), k, v))
    want, mag = ref.attention(q1, k1, v1, [n], [n], causal=True)
    ref.check_attention(B.attention(q1, k1, v1, ints([0, n]), ints([0, n]), n, n, causal=True), want, mag, "one head")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(300, 700, 640), (300, 700, 128), (2100, 700, 272), (3333, 1203, 656), (4352, 4096, 1152), (4097, 4200, 1408)])
def test_scales_that_end_inside_16_bytes(m, n, k, dtype):
    """Row scales 4 a load, of rows that end inside one: what lies behind a row's last scale is never used."""
    say(f"scaled product with padded row scales {m} x {n} x {k} {dtype}")
    kb = -(-k // 128)
    x, w, ws = bits8(m, k, 61), bits8(n, k, 62), scales(-(-n // 128), k, 64) * 1e-4
    wide = torch.full((m, -(-kb // 4) * 4), float("nan"), device=DEV)
    wide[:, :kb] = scales(m, k, 63) * 1e-4
    xs = wide[:, :kb]
    assert xs.stride(0) % 4 == 0 and kb % 4 != 0
    want, mag = ref.scaled_linear(x, xs, w, ws)
    ref.check_linear(B.scaled_linear(x, xs, w, ws, dtype, exact=True), want, mag, k, "padded scales")
    # as scales without gaps, loaded one by one
    assert torch.equal(B.scaled_linear(x, xs, w, ws, dtype), B.scaled_linear(x, xs.contiguous(), w, ws, dtype))
