"""spconv_rms_norm against the formula in 64 bits: types, widths, strides, 8-bit rows."""
from __future__ import annotations

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests import transformer_ref as ref
from tests.gpu_helpers import DEV, say

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def rows(n, c, dtype, seed, pad=0, shift=0):
    """Rows of different sizes in a wider array, `shift` elements into it."""
    g = torch.Generator(DEV).manual_seed(seed)
    flat = torch.randn(n * (c + pad) + shift, device=DEV, generator=g).to(dtype)
    x = flat[shift:].view(n, c + pad)
    x *= torch.exp(torch.randn((n, 1), device=DEV, generator=g)).to(dtype)
    return x[:, :c]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,c,pad,shift", [
    (1, 1, 0, 0), (3, 8, 0, 0), (1, 16, 0, 0), (5, 120, 8, 0), (1000, 128, 0, 0), (77, 136, 0, 0), (64, 256, 16, 0),
    (33, 264, 0, 8), (9, 512, 0, 0), (7, 1000, 536, 0), (2, 1024, 0, 0), (4, 2048, 0, 0), (3, 4096, 0, 0),
    (2, 4104, 0, 0), (2, 8192, 0, 0), (1, 16384, 0, 0), (2, 16400, 0, 0), (5, 7, 0, 0), (4, 129, 3, 0), (6, 256, 0, 1),
])
def test_norm(n, c, pad, shift, dtype):
    say(f"norm {n} x {c} {dtype}, pad {pad}, shift {shift}")
    x, res = rows(n, c, dtype, 1, pad, shift), rows(n, c, dtype, 2)
    gamma = (1 + 0.2 * torch.randn(c, device=DEV)).to(dtype)
    y, scale, total = B.rms_norm(x, gamma)
    assert scale is None and total is None
    want, _ = ref.rms_norm(x, gamma)
    ref.check_rows(y, want, c, "norm")
    y, _, total = B.rms_norm(x, gamma, residual=res)
    want, s = ref.rms_norm(x, gamma, res)
    # the norm is that of the sum in float32
    ref.check_rows(total, s, 16, "sum")
    mag = x.double().abs() + res.double().abs()
    off, slack = (y.double() - want).abs(), (want / s.where(s != 0, 1.0)).abs() * mag * 2.0 ** -23
    bound = want.abs() * (ref.UNIT[dtype] + (c / 16 + 16) * 2.0 ** -24) + slack + ref.TINY[dtype]
    assert bool((off <= bound).all())
    if c % 16 == 0:
        q, scale, total8 = B.rms_norm(x, gamma, bits8=True)
        want, _ = ref.rms_norm(x, gamma)
        ref.check_bits8(q, scale, want, "8 bits")
        q2, scale2, total8 = B.rms_norm(x, gamma, residual=res, bits8=True)
        assert torch.equal(total8, total)


def test_norm_repeats_to_the_bit():
    say("norm, repeated")
    x, res = rows(501, 768, torch.bfloat16, 5), rows(501, 768, torch.bfloat16, 6)
    gamma = torch.ones(768, device=DEV, dtype=torch.bfloat16)
    a = B.rms_norm(x, gamma, residual=res, bits8=True)
    b = B.rms_norm(x, gamma, residual=res, bits8=True)
    assert all(torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(a, b))


def test_norm_of_no_rows_and_of_zeros():
    say("norm of no rows, of zeros")
    gamma = torch.ones(256, device=DEV, dtype=torch.float16)
    y, scale, _ = B.rms_norm(torch.empty((0, 256), device=DEV, dtype=torch.float16), gamma, bits8=True)
    assert y.shape == (0, 256) and scale.shape == (0, 2)
    y, scale, _ = B.rms_norm(torch.zeros((3, 256), device=DEV, dtype=torch.float16), gamma, bits8=True)
    assert bool((y.float() == 0).all()) and bool((scale == 2.0 ** -126).all())


@pytest.mark.parametrize("c", [256, 1296])
def test_norm_not_a_number_stays_in_its_row(c):
    say("norm with NaN and infinity")
    x = rows(6, c, torch.float32, 7).contiguous()
    gamma = torch.ones(c, device=DEV)
    clean, _, _ = B.rms_norm(x, gamma)
    x[1, 5], x[4, c - 1] = float("nan"), float("inf")
    y, _, _ = B.rms_norm(x, gamma)
    q, scale, _ = B.rms_norm(x, gamma, bits8=True)
    assert bool(y[1].isnan().all()) and bool(q[1].float().isnan().all())
    # an infinite mean square: the other elements are 0, its own is not a number
    assert bool((y[4, :-1] == 0).all()) and bool(y[4, -1].isnan()) and bool(q[4, -1].float().isnan())
    keep = [0, 2, 3, 5]
    assert torch.equal(y[keep], clean[keep])


def test_sum_in_place():
    """The sum may be stored over x or over the residual."""
    say("norm, sum in place")
    for c in (512, 515):
        x, res = rows(37, c, torch.float16, 8).contiguous(), rows(37, c, torch.float16, 9).contiguous()
        gamma = torch.ones(c, device=DEV, dtype=torch.float16)
        want, _, total = B.rms_norm(x, gamma, residual=res)
        for target in (0, 1):
            a, b = x.clone(), res.clone()
            y = torch.empty_like(x)
            B.spconv_rms_norm(a, b, gamma, (a, b)[target], y, None, 1e-6)
            assert torch.equal((a, b)[target], total) and torch.equal(y, want)


def test_norm_on_another_stream():
    say("norm on another stream")
    x = rows(4000, 1024, torch.bfloat16, 10)
    gamma = torch.ones(1024, device=DEV, dtype=torch.bfloat16)
    want, _, _ = B.rms_norm(x, gamma)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y, _, _ = B.rms_norm(x, gamma, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,c,pad,shift", [(37, 2, 0, 0), (35, 100, 0, 0), (18, 192, 1, 0), (19, 193, 0, 0), (7, 640, 0, 3),
                                           (5, 641, 0, 0), (3, 4097, 0, 0), (7, 96, 0, 1), (9, 784, 0, 1)])
def test_norm_of_any_width(n, c, pad, shift, dtype):
    """Rows that no wide access fits, by as many lanes as their width asks for."""
    say(f"norm of any width {n} x {c} {dtype}, pad {pad}, shift {shift}")
    x, gamma = rows(n, c, dtype, 11, pad, shift), (1 + 0.2 * torch.randn(c, device=DEV)).to(dtype)
    y, _, _ = B.rms_norm(x, gamma)
    want, _ = ref.rms_norm(x, gamma)
    ref.check_rows(y, want, c, "norm")
    _, _, total = B.rms_norm(x, gamma, residual=x)
    assert torch.equal(total, x + x)
    if c % 16 == 0:
        ref.check_bits8(*B.rms_norm(x, gamma, bits8=True)[:2], want, "8 bits")
