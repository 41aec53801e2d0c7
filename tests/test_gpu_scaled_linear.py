"""spconv_scaled_linear against the product in 64 bits."""
from __future__ import annotations

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests import transformer_ref as ref
from tests.gpu_helpers import DEV, say

pytestmark = pytest.mark.gpu


def bits8(n, c, seed, pad=0):
    """e4m3 rows of all kinds of values (subnormal ones and 448 among them) and scales over a wide range."""
    g = torch.Generator(DEV).manual_seed(seed)
    codes = torch.randint(0, 256, (n, c + pad), device=DEV, generator=g, dtype=torch.int32)
    codes = torch.where(codes % 128 == 127, codes - 1, codes).to(torch.uint8)  # 0x7f and 0xff are NaN
    return codes.view(torch.float8_e4m3fn)[:, :c]


def scales(rows, k, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    return torch.exp2(2 * torch.randn((rows, -(-k // 128)), device=DEV, generator=g))


SHAPES = [(1, 1, 16), (1, 16, 128), (1, 4096, 1024), (2, 100, 144), (16, 48, 256), (17, 130, 1008), (33, 1001, 4096),
          (64, 257, 640), (65, 128, 128), (100, 129, 16), (128, 128, 256), (129, 300, 400), (300, 77, 2048),
          (1000, 768, 256), (513, 1024, 4096), (2049, 260, 144), (5000, 96, 32), (700, 2500, 1040)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear(m, n, k, dtype):
    say(f"scaled product {m} x {n} x {k} {dtype}")
    x, w = bits8(m, k, 1), bits8(n, k, 2)
    xs, ws = scales(m, k, 3) * 1e-4, scales(-(-n // 128), k, 4) * 1e-4
    want, mag = ref.scaled_linear(x, xs, w, ws)
    ref.check_linear(B.scaled_linear(x, xs, w, ws, dtype, exact=True), want, mag, k, "product")
    ref.check_linear(B.scaled_linear(x, xs, w, ws, dtype, relu=True, exact=True), want.relu(), mag, k, "product with ReLU")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear_by_the_8_bit_instruction(m, n, k, dtype):
    """Without ``exact``, in 16-bit types: of each group of eight products, up to seven may be dropped
    that are 2^13 times smaller than the largest, so 7 2^-13 of the sum of magnitudes at most."""
    say(f"scaled product by the 8-bit instruction {m} x {n} x {k} {dtype}")
    x, w = bits8(m, k, 1), bits8(n, k, 2)
    xs, ws = scales(m, k, 3) * 1e-4, scales(-(-n // 128), k, 4) * 1e-4
    want, mag = ref.scaled_linear(x, xs, w, ws)
    got = B.scaled_linear(x, xs, w, ws, dtype)
    bound = mag * (7 * 2.0 ** -13 + (min(k, 128) + k / 128 + 4) * 2.0 ** -24) + want.abs() * ref.UNIT[dtype] + ref.TINY[dtype]
    assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("m", [1, 40, 300])
def test_linear_strides(m):
    """Rows inside wider rows, scales too, and an output inside wider rows that stay as they are."""
    say(f"scaled product, strided, {m} rows")
    n, k = 200, 272
    x, w = bits8(m, k, 5, pad=48), bits8(n, k, 6, pad=16)
    xs, ws = scales(m, k + 512, 7)[:, 1:4] * 1e-4, scales(2, k + 256, 8)[:, 2:5] * 1e-4
    want, mag = ref.scaled_linear(x, xs, w, ws)
    for pad, first in ((8, 0), (3, 1), (8, 8)):
        wide = torch.full((m, n + pad + first), 7.0, device=DEV, dtype=torch.float16)
        B.spconv_scaled_linear(x, xs, w, ws, wide[:, first:first + n], exact=True)
        ref.check_linear(wide[:, first:first + n], want, mag, k, "strided")
        assert bool((wide[:, :first] == 7).all()) and bool((wide[:, first + n:] == 7).all())


def test_linear_without_columns_or_rows():
    say("scaled product without columns")
    x, w = bits8(5, 0, 1), bits8(70, 0, 2)
    y = B.scaled_linear(x, scales(5, 0, 3), w, scales(1, 0, 4), torch.float32)
    assert y.shape == (5, 70) and bool((y == 0).all())
    assert B.scaled_linear(bits8(0, 64, 1), scales(0, 64, 3), bits8(9, 64, 2), scales(1, 64, 4), torch.float32).shape == (0, 9)


@pytest.mark.parametrize("m", [3, 200])
def test_linear_not_a_number_stays_in_its_row(m):
    say("scaled product with NaN and infinite scales")
    n, k = 150, 384
    x, w = bits8(m, k, 9).clone(), bits8(n, k, 10)
    xs, ws = scales(m, k, 11), scales(2, k, 12)
    clean = B.scaled_linear(x, xs, w, ws, torch.float32)
    x.view(torch.uint8)[1, 130] = 0x7F
    xs[2, 0] = float("inf")
    y = B.scaled_linear(x, xs, w, ws, torch.float32)
    assert bool(y[1].isnan().all()) and not bool(y[2].isfinite().any())
    keep = [i for i in range(m) if i not in (1, 2)]
    assert torch.equal(y[keep], clean[keep])


def test_linear_reads_what_the_norm_writes():
    say("norm, then product")
    g = torch.Generator(DEV).manual_seed(13)
    x = torch.randn((333, 512), device=DEV, generator=g).to(torch.bfloat16)
    q, scale, _ = B.rms_norm(x, torch.ones(512, device=DEV, dtype=torch.bfloat16), bits8=True)
    w = torch.randn((640, 512), device=DEV, generator=g) / 512 ** 0.5
    wq, ws = B.quantize_weight(w)
    y = B.scaled_linear(q, scale, wq, ws, torch.bfloat16)
    want, mag = ref.scaled_linear(q, scale, wq, ws)
    ref.check_linear(y, want, mag, 512, "product")
    full = ref.rms_norm(x, torch.ones(512, device=DEV))[0] @ w.double().t().contiguous()
    # two operands rounded to 4 significant bits: 2^-4 / sqrt(3) each, as a root mean square at most
    assert float((y.double() - full).norm() / full.norm()) < 2 * 2.0 ** -4 / 3 ** 0.5


def test_quantized_weights():
    say("weights in 8 bits")
    g = torch.Generator(DEV).manual_seed(14)
    w = torch.randn((200, 300), device=DEV, generator=g)
    w[:128, :128] = 0
    q, s = B.quantize_weight(w)
    assert q.shape == (200, 300) and s.shape == (2, 3) and float(s[0, 0]) == 2.0 ** -126
    f = s.double().repeat_interleave(128, 0)[:200].repeat_interleave(128, 1)[:, :300]
    step = torch.maximum(w.double().abs() * 2.0 ** -4, f * 2.0 ** -10)
    assert bool(((q.float().double() * f - w.double()).abs() <= step * (1 + 2.0 ** -10)).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(4100, 4200, 272), (4352, 4096, 1152), (8191, 2100, 640)])
def test_linear_of_many_tiles(m, n, k, dtype):
    """Large products take tiles of 256 x 256."""
    say(f"scaled product {m} x {n} x {k} {dtype}")
    x, w = bits8(m, k, 21), bits8(n, k, 22)
    xs, ws = scales(m, k, 23) * 1e-4, scales(-(-n // 128), k, 24) * 1e-4
    want, mag = ref.scaled_linear(x, xs, w, ws)
    got = B.scaled_linear(x, xs, w, ws, dtype)
    bound = mag * (7 * 2.0 ** -13 + (min(k, 128) + k / 128 + 4) * 2.0 ** -24) + want.abs() * ref.UNIT[dtype] + ref.TINY[dtype]
    assert bool(((got.double() - want).abs() <= bound).all())
    ref.check_linear(B.scaled_linear(x, xs, w, ws, dtype, exact=True), want, mag, k, "exact")


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("first", [0, 1, 8])
@pytest.mark.parametrize("m,n,k", [(333, 200, 272), (333, 136, 1152), (200, 3, 640), (4200, 4203, 1152)])
def test_linear_stores_only_its_outputs(m, n, k, dtype, first):
    """Outputs inside wider rows of any alignment, of numbers that fill no 16 bytes."""
    say(f"scaled product into a part of wider rows, {m} x {n} x {k} {dtype} from {first}")
    x, w = bits8(m, k, 31), bits8(n, k, 32)
    xs, ws = scales(m, k, 33) * 1e-4, scales(-(-n // 128), k, 34) * 1e-4
    want = B.scaled_linear(x, xs, w, ws, dtype)
    for pad in (5, 8):
        wide = torch.full((m + 1, first + n + pad), 7.0, device=DEV, dtype=dtype)
        B.spconv_scaled_linear(x, xs, w, ws, wide[:m, first:first + n])
        assert torch.equal(wide[:m, first:first + n], want)
        wide[:m, first:first + n] = 7.0
        assert bool((wide == 7).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(1, 4112, 2064), (20, 4200, 272), (40, 4111, 640), (64, 5000, 144), (33, 4097, 1536),
                                   (64, 1024, 4096), (128, 1000, 3200), (250, 1024, 4096)])
def test_linear_of_few_rows_and_many_outputs(m, n, k, dtype):
    say(f"scaled product {m} x {n} x {k} {dtype}")
    x, w = bits8(m, k, 41), bits8(n, k, 42)
    xs, ws = scales(m, k, 43) * 1e-4, scales(-(-n // 128), k, 44) * 1e-4
    want, mag = ref.scaled_linear(x, xs, w, ws)
    ref.check_linear(B.scaled_linear(x, xs, w, ws, dtype, exact=True), want, mag, k, "product")


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(2100, 700, 272), (2100, 703, 1040), (3333, 1203, 144), (3333, 1200, 656), (2500, 3001, 272),
                                   (2500, 3001, 784), (9000, 17, 528), (70, 4000, 256)])
def test_linear_of_tiles_of_all_sizes(m, n, k, dtype):
    """Against the product, and outputs inside wider rows that stay as they are."""
    say(f"scaled product by tiles {m} x {n} x {k} {dtype}")
    x, w = bits8(m, k, 51), bits8(n, k, 52)
    xs, ws = scales(m, k, 53) * 1e-4, scales(-(-n // 128), k, 54) * 1e-4
    want, mag = ref.scaled_linear(x, xs, w, ws)
    ref.check_linear(B.scaled_linear(x, xs, w, ws, dtype, exact=True), want, mag, k, "product")
    got = B.scaled_linear(x, xs, w, ws, dtype, relu=True)
    bound = mag * (7 * 2.0 ** -13 + (min(k, 128) + k / 128 + 4) * 2.0 ** -24) + want.abs() * ref.UNIT[dtype] + ref.TINY[dtype]
    assert bool(((got.double() - want.relu()).abs() <= bound).all())
    for first, pad in ((0, 5), (8, 8)):
        wide = torch.full((m + 1, first + n + pad), 7.0, device=DEV, dtype=dtype)
        B.spconv_scaled_linear(x, xs, w, ws, wide[:m, first:first + n], relu=True)
        assert torch.equal(wide[:m, first:first + n], got)
        wide[:m, first:first + n] = 7.0
        assert bool((wide == 7).all())
