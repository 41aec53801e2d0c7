"""spconv_rms_norm where test_gpu_norm.py does not look: 8-bit rows of a sum, and the ends of what it accepts."""
from __future__ import annotations

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests import transformer_ref as ref
from tests.gpu_helpers import DEV, say
from tests.test_gpu_norm import DTYPES, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,c,pad,shift", [
    (3, 16, 0, 0), (1000, 128, 0, 0), (77, 144, 0, 0), (64, 256, 16, 0), (9, 512, 0, 0), (7, 1008, 536, 0), (1, 1024, 0, 0),
    (4, 2048, 0, 0), (3, 4096, 0, 0), (2, 8192, 0, 0), (2, 16400, 0, 0), (6, 256, 0, 1), (18, 192, 1, 0), (9, 784, 0, 1),
])
def test_8_bit_rows_of_a_sum(n, c, pad, shift, dtype):
    """Values and scales of the norm of x + residual, by whole accesses and element by element."""
    say(f"norm of a sum in 8 bits {n} x {c} {dtype}, pad {pad}, shift {shift}")
    x, res = rows(n, c, dtype, 1, pad, shift), rows(n, c, dtype, 2)
    gamma = (1 + 0.2 * torch.randn(c, device=DEV)).to(dtype)
    q, scale, total = B.rms_norm(x, gamma, residual=res, bits8=True)
    want, s = ref.rms_norm(x, gamma, res)
    ref.check_rows(total, s, 16, "sum")
    # where x and the residual cancel, the rounding of their float32 sum counts, once at their size
    cancel = (want / s.where(s != 0, 1.0)).abs() * (x.double().abs() + res.double().abs()) * 2.0 ** -23
    slack = (c / 16 + 16) * 2.0 ** -24
    exact_top = (ref.block_top(want) / 448.0).clamp(min=2.0 ** -126)
    scale_slack = exact_top * (slack + 2.0 ** -23) + ref.block_top(cancel) / 448.0
    assert bool(((scale.double() - exact_top).abs() <= scale_slack).all())
    step = torch.maximum(want.abs() * 2.0 ** -4, ref.spread(scale, c) * 2.0 ** -10)
    off = (q.float().double() * ref.spread(scale, c) - want).abs()
    assert bool((off <= step * (1 + 2.0 ** -10) + want.abs() * slack + cancel).all())


@pytest.mark.parametrize("c,residual,bits8", [(1032, False, False), (1040, False, True), (641, True, False)])
def test_more_rows_than_one_launch_takes(c, residual, bits8):
    """2^24 rows and more, each by a workgroup of 256 threads: 2^32 threads and more."""
    say(f"norm of 16.8 million rows of {c}")
    few, times = 4099, 4100  # a prime number of rows, again and again
    assert few * times > 1 << 24
    dtype = torch.float16
    x, gamma = rows(few, c, dtype, 12).contiguous(), (1 + 0.2 * torch.randn(c, device=DEV)).to(dtype)
    want = B.rms_norm(x, gamma, residual=x if residual else None, bits8=bits8)
    wide = x.repeat(times, 1)
    got = B.rms_norm(wide, gamma, residual=wide if residual else None, bits8=bits8)
    for a, b in zip(got, want):
        if b is None:
            assert a is None
            continue
        a, b = (t.view(torch.uint8) if t.dtype == B.E4M3 else t for t in (a, b))
        for part in a.view(times, few, -1).split(100):
            assert bool((part == b).all())
    del wide, got, a, part
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("c,shift", [(256, 0), (1296, 0), (256, 1), (16400, 0)])
def test_a_block_with_an_infinity(c, shift, dtype):
    """A block with an infinite value has an infinite scale and stands for NaN; others are as without it."""
    say(f"norm in 8 bits with an infinite gamma, {c} columns {dtype}")
    x = rows(5, c, dtype, 13, 0, shift)
    x[x == 0] = 1.0
    gamma = (1 + 0.2 * torch.randn(c, device=DEV)).to(dtype)
    want, want_scale, _ = B.rms_norm(x, gamma, bits8=True)
    gamma[130] = float("inf")
    q, scale, _ = B.rms_norm(x, gamma, bits8=True)
    y = B.rms_norm(x, gamma)[0]
    assert bool(y[:, 130].isinf().all())
    hit = torch.zeros(c, dtype=torch.bool, device=DEV)
    hit[128:256] = True
    assert bool((scale[:, 1] == float("inf")).all()) and bool(q.float()[:, hit].isnan().all())
    assert torch.equal(q.float()[:, ~hit], want.float()[:, ~hit])
    keep = [i for i in range(scale.shape[1]) if i != 1]
    assert torch.equal(scale[:, keep], want_scale[:, keep])
