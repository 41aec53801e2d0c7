"""Values that are no finite numbers, over pages: at every key of a tile, in the first and last columns, in forms whose
rows in LDS are wider than the heads."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests.cache_ref import Cached
from tests.gpu_helpers import DEV, say

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HEADS, KV = 4, 2
QL, KL = [100, 70], [200, 170]  # of the first document's keys 100 .. 199 are seen by some queries and not by others


def documents(d, dtype, bits8, ql=QL):
    return Cached(ql, KL, HEADS, KV, d, dtype, bits8, 16, seed=d)


def row_of(b, place):
    """(page, row) of a key of the first document."""
    return int(b.table[0, place // 16]), place % 16


def check(b, clean, place, head, columns, is_value):
    """Queries of document 0 from `place` on, in the heads of a key head, get the value in these columns; all else has
    the bits it had."""
    got = b.run()
    sees = torch.zeros(got.shape, dtype=torch.bool, device=DEV)
    group = HEADS // KV
    queries = b.q_lens[0]
    first = queries - (KL[0] - place)
    sees[max(first, 0):queries, head * group:(head + 1) * group, columns] = True
    assert bool(is_value(got[sees]).all()), f"key {place}: a query that sees it has not got its value"
    other = got[~sees]
    assert torch.equal(other, clean[~sees]), (f"key {place}: {int((other != clean[~sees]).sum())} values of "
                                              "queries or columns that it is no part of have changed")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("d", [16, 80, 96, 128])
def test_a_nan_of_8_bits_at_every_key_of_a_tile(d, dtype):
    """One NaN byte in a value's last columns."""
    b = documents(d, dtype, True)
    clean = b.run()
    v = b.cache.v.view(torch.uint8)
    for place in range(128, 192):
        say(f"8 bits, {d} columns {dtype}: NaN at key {place}")
        page, row = row_of(b, place)
        column = d - 1 - place % 16
        kept = int(v[page, 1, row, column])
        v[page, 1, row, column] = 0x7f
        check(b, clean, place, 1, column, torch.isnan)
        v[page, 1, row, column] = kept


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("d", [80, 96])
@pytest.mark.parametrize("scale", [math.nan, math.inf])
def test_scales_that_are_not_finite(scale, d, dtype):
    """They make their row NaN, and no other."""
    b = documents(d, dtype, True)
    clean = b.run()
    for place in (128, 131, 158, 159, 160, 190, 191, 199):
        say(f"8 bits, {d} columns {dtype}: scale {scale} at key {place}")
        page, row = row_of(b, place)
        kept = float(b.cache.v_scale[page, 0, row])
        b.cache.v_scale[page, 0, row] = scale
        check(b, clean, place, 0, slice(None), torch.isnan)
        b.cache.v_scale[page, 0, row] = kept


@pytest.mark.parametrize("d", [80, 96])
@pytest.mark.parametrize("sign", [1, -1])
def test_8_bits_beyond_float16(sign, d):
    """A value that float16 cannot hold is an infinity there, to the queries that see it."""
    b = documents(d, F16, True)
    v = b.cache.v.view(torch.uint8)
    for place in (128, 159, 190, 191):
        page, row = row_of(b, place)
        v[page, 1, row] = 0
        b.cache.v_scale[page, 1, row] = 256.0
        clean = b.run()
        for column in (0, 31, 32, d - 16, d - 1):
            say(f"8 bits of float16, {d} columns: {sign * 448 * 256} at key {place}, column {column}")
            v[page, 1, row, column] = 0x7e if sign > 0 else 0xfe
            check(b, clean, place, 1, column, lambda x: x == sign * math.inf)
            v[page, 1, row, column] = 0


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("d", [72, 80, 96])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_pages_of_the_rows_type(value, d, dtype):
    b = documents(d, dtype, False)
    clean = b.run()
    for place in (128, 158, 159, 190, 191, 199):
        for column in (0, d - 16, d - 1):
            say(f"{d} columns {dtype}: {value} at key {place}, column {column}")
            page, row = row_of(b, place)
            kept = b.cache.v[page, 1, row, column].clone()
            b.cache.v[page, 1, row, column] = value
            check(b, clean, place, 1, column, torch.isnan if math.isnan(value) else lambda x: x == value)
            b.cache.v[page, 1, row, column] = kept


def test_packed_keys():
    """The same over keys in one run of memory."""
    for d in (72, 96):
        b = documents(d, BF16, False)
        k, v = b.k.to(BF16), b.v.to(BF16)
        start = torch.tensor([0, KL[0], sum(KL)], dtype=torch.int32, device=DEV)

        def run(v):
            return B.attention(b.q, k, v, b.q_start, start, max(QL), max(KL), causal=True)

        clean = run(v)
        for place in (128, 190, 191):
            say(f"packed, {d} columns: NaN at key {place}")
            w = v.clone()
            w[place, 1, d - 1] = math.nan
            b.run = lambda: run(w)
            check(b, clean, place, 1, d - 1, torch.isnan)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("d", [16, 48, 80, 96, 128, 256])
def test_few_queries(d, bits8, dtype):
    """Five new tokens: each sees its own place and those before."""
    b = documents(d, dtype, bits8, ql=[5, 1])
    clean = b.run()
    v = b.cache.v.view(torch.uint8) if bits8 else b.cache.v
    for place in range(190, 200):
        for column in (0, d // 2 + 3, d - 1):
            say(f"few queries, 8 bits {bits8}, {d} columns {dtype}: NaN at key {place}, column {column}")
            page, row = row_of(b, place)
            kept = v[page, 1, row, column].clone()
            v[page, 1, row, column] = 0x7f if bits8 else math.nan
            check(b, clean, place, 1, column, torch.isnan)
            v[page, 1, row, column] = kept


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("n", [2000, 5000, 40_000])
def test_a_nan_of_no_weight(n, dtype):
    """A value that is seen with a weight below float32's least number: 0 times NaN is NaN, however many ranges of keys
    a row is joined from (1 to 8, more, and more than a wave has lanes)."""
    say(f"one token of {n} keys {dtype}: a NaN of no weight")
    d = 64
    k = torch.zeros((n, 1, d), device=DEV)
    k[:n // 3, :, 0] = -300.0  # whole ranges
    b = Cached([1], [n], 2, 1, d, dtype, False, 16, seed=n % 97, like=(k, torch.randn((n, 1, d), device=DEV)))
    b.q[:] = 0.0
    b.q[..., 0] = 1.0
    start = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    packed_k, packed_v = b.k.to(dtype), b.v.to(dtype)

    def both():
        return (b.run(scale=1.0), B.attention(b.q, packed_k, packed_v, b.q_start, start, 1, n, causal=True, scale=1.0))

    clean = both()
    page, row = row_of(b, 3)
    b.cache.v[page, 0, row, 5] = math.nan
    packed_v[3, 0, 5] = math.nan
    for got, was, what in zip(both(), clean, ("pages", "packed keys")):
        assert bool(got[..., 5].isnan().all()), what
        got[..., 5] = was[..., 5]
        assert torch.equal(got, was), what
