"""spconv_cache_write and spconv_cache_read: tokens into pages and back, against 64 bits."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests import cache_ref as cref
from tests import transformer_ref as ref
from tests.gpu_helpers import DEV, say

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


def rows_of(b, t, name):
    """What document t's pages hold: (rows [n][heads][d], scales or None)."""
    place = torch.arange(b.k_lens[t], device=DEV)
    at = b.table[t].long()[place // b.page]
    x, s = getattr(b.cache, name), getattr(b.cache, name + "_scale")
    got = x.view(torch.uint8)[at, :, place % b.page].view(B.E4M3) if b.bits8 else x[at, :, place % b.page]
    return got, None if s is None else s[at, :, place % b.page]


def bits(t):
    return t.contiguous().view(torch.uint8)


SHAPES = [(1, 64, 16), (2, 32, 8), (8, 128, 64), (3, 80, 1), (1, 256, 128), (5, 16, 32), (2, 96, 16)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("kv,d,page", SHAPES)
def test_write_and_read(kv, d, page, bits8, dtype):
    say(f"cache of {kv} heads of {d}, pages of {page}, 8 bits {bits8}, {dtype}")
    for new, kl in (([1], [1]), ([1, 1, 1, 1], [5, 1, 0, 70]), ([3, 0, 40, 17], [3, 9, 100, 17]), ([700, 260], [700, 1300])):
        new = [min(a, b) for a, b in zip(new, kl)]
        b = cref.Cached(new, kl, kv, kv, d, dtype, bits8, page, seed=d + page)
        before = {n: bits(getattr(b.cache, n)).clone() for n in ("k", "v")}
        g = torch.Generator(DEV).manual_seed(1)
        fused = (torch.randn((sum(new), 3 * kv * d), device=DEV, generator=g)
                 * torch.exp(2 * torch.randn((sum(new), 1), device=DEV, generator=g))).to(dtype)
        _, k, v = (t.unflatten(1, (-1, d)) for t in fused.split([kv * d] * 3, 1))
        B.cache_write(b.cache, k, v, b.q_start, b.k_len, b.table)
        at = 0
        used = torch.zeros(before["k"].shape[:3], dtype=torch.bool, device=DEV)
        for t, (m, n) in enumerate(zip(new, kl)):
            for name, x in (("k", k), ("v", v)):
                got, scale = rows_of(b, t, name)
                mine = x[at:at + m]
                if bits8:
                    cref.check_rows8(got[n - m:], scale[n - m:], mine, f"document {t}")
                else:
                    assert torch.equal(got[n - m:], mine), f"document {t}"
                # the document's earlier rows are what they were
                held = (b.k if name == "k" else b.v)[sum(kl[:t]):sum(kl[:t]) + n - m]
                old = got[:n - m].double() if not bits8 else got[:n - m].float().double() * scale[:n - m].double()[..., None]
                assert torch.equal(old, held)
            place = torch.arange(n - m, n, device=DEV)
            used[b.table[t].long()[place // page], :, place % page] = True
            at += m
        for name in ("k", "v"):  # and nothing else was written
            now = bits(getattr(b.cache, name))
            assert torch.equal(now[~used], before[name][~used])
        rows = sum(kl)
        got = B.cache_read(b.cache, cref.starts(kl), b.table, rows, dtype)
        for t, n in enumerate(kl):
            for name, x in zip("kv", got):
                held, scale = rows_of(b, t, name)
                want = held.double() if not bits8 else held.float().double() * scale.double()[..., None]
                mine = x[sum(kl[:t]):sum(kl[:t]) + n]
                assert mine.dtype == dtype
                if bits8:
                    off = (mine.double() - want).abs()
                    assert bool((off <= want.abs() * (ref.UNIT[dtype] + 2.0 ** -24) + ref.TINY[dtype]).all())
                else:
                    assert torch.equal(mine, held)


@pytest.mark.parametrize("dtype", TYPES)
def test_rounding_of_8_bits(dtype):
    """Every e4m3 number and the middles between them keep their place; rows of zeros, of the type's
    smallest and largest numbers."""
    say(f"8-bit rows at their borders {dtype}")
    every = torch.arange(256, dtype=torch.uint8).view(B.E4M3).float()
    every = every[every.isfinite()]
    values = torch.cat([every, every])[:256 - 16].to(DEV)
    x = torch.zeros((6, 1, 256), device=DEV)
    x[0, 0, :240], x[0, 0, 240] = values, 448.0           # scale 1: exact
    x[1, 0, :240], x[1, 0, 240] = values / 64, 7.0        # a power of two
    x[2] = torch.finfo(dtype).max if dtype != BF16 else 3e38
    x[3] = torch.finfo(dtype).tiny
    x[4] = torch.linspace(-1, 1, 256, device=DEV)
    x = x.to(dtype)
    c = B.Pages.make(2, 8, 1, 256, dtype, True, DEV)
    table = cref.ints([[1]])
    B.cache_write(c, x, -x, cref.starts([6]), cref.ints([6]), table)
    q, s = c.k.view(torch.uint8)[1, 0, :6].view(B.E4M3), c.k_scale[1, 0, :6]
    cref.check_rows8(q, s, x[:, 0], "keys")
    assert float(s[0]) == 1.0 and torch.equal(q[0, :240].float(), values) and float(s[5]) == 2.0 ** -126
    assert torch.equal(q[1, :240].float(), values) and float(s[1]) == 2.0 ** -6
    assert torch.equal(c.v.view(torch.uint8)[1, 0, :6].view(B.E4M3).float(), -q.float())
    k, v = B.cache_read(c, cref.starts([6]), table, 6, dtype)
    assert bool(k.isfinite().all()) and torch.equal(k, -v) and torch.equal(k[0], x[0])


def test_odd_values():
    """NaN stays NaN, and alone; an infinity makes its row NaN, and no other."""
    say("8-bit rows with NaN and infinities")
    x = torch.randn((5, 2, 32), device=DEV)
    x[1, 0, 3], x[2, 1, 7] = math.nan, -math.inf
    c = B.Pages.make(3, 2, 2, 32, F32, True, DEV)
    table = cref.ints([[2, 0, 1]])
    B.cache_write(c, x, x, cref.starts([5]), cref.ints([5]), table)
    k, v = B.cache_read(c, cref.starts([5]), table, 5, F32)
    for y in (k, v):
        bad = y.isnan()
        assert bool(bad[1, 0, 3]) and int(bad[1].sum()) == 1 and bool(bad[2, 1].all()) and int(bad.sum()) == 33


def test_pages_that_are_none():
    """Entries outside the pages, places before 0 and behind the table: nothing is written there, and
    zeros are read; rows of no document are left as they are."""
    say("cache calls beyond the pages")
    for bits8 in (False, True):
        c = B.Pages.make(4, 8, 2, 32, BF16, bits8, DEV)
        held = bits(c.k).clone()
        table = cref.ints([[-1, 4], [1 << 30, -(1 << 31)], [3, 2]])
        # two rows before the first document, eight of each, and three behind the last
        start = cref.ints([2, 10, 18, 26])
        x = torch.randn((29, 2, 32), device=DEV).to(BF16)
        B.cache_write(c, x, x, start, cref.ints([8, 16, 20]), table)   # document 2: places 12 .. 19, 16 on behind the table
        now = bits(c.k)
        changed = (now != held).flatten(2).any(2).any(1)
        assert changed.tolist() == [False, False, True, False]
        B.cache_write(c, x, x, start, cref.ints([8, 16, 3]), table)    # places -5 .. 2
        changed = (bits(c.k) != held).flatten(2).any(2).any(1)
        assert changed.tolist() == [False, False, True, True]
        # the C call, on outputs that are set before
        k, v = (torch.full((29, 2, 32), 7.0, device=DEV).to(BF16) for _ in range(2))
        p = pages_args(c, table)
        B.spconv_cache_read(p, k, v, start)
        for y in (k, v):
            assert bool((y[:2] == 7).all()) and bool((y[26:] == 7).all()) and bool((y[2:18] == 0).all())
        long = cref.ints([0, 0, 0, 29])  # the third document alone, longer than its table
        B.spconv_cache_read(p, k, v, long)
        assert bool((k[16:] == 0).all()) and bool((k[:3] != 0).any()) and bool((k[12:16] != 0).any())


def pages_args(c, table):
    return B.PagesArgs(d_k=c.k.data_ptr(), d_v=c.v.data_ptr(), d_k_scale=c.k_scale.data_ptr() if c.k_scale is not None else None,
                       d_v_scale=c.v_scale.data_ptr() if c.v_scale is not None else None, d_table=table.data_ptr(),
                       n_pages=c.k.shape[0], n_docs=table.shape[0], table_row=table.shape[1], page=c.page,
                       kv_heads=c.k.shape[1], head_dim=c.k.shape[3])


def test_many_documents():
    """More documents than are looked through in LDS, most of them empty."""
    say("cache of 3000 documents")
    lens = [(i * 7) % 5 if i % 3 == 0 else 0 for i in range(3000)]
    n = sum(lens)
    c = B.Pages.make(3000, 4, 1, 16, F32, False, DEV)
    table = torch.randperm(3000, device=DEV).to(torch.int32)[:, None].contiguous()
    x = torch.randn((n, 1, 16), device=DEV)
    B.cache_write(c, x, 2 * x, cref.starts(lens), cref.ints(lens), table)
    k, v = B.cache_read(c, cref.starts(lens), table, n, F32)
    assert torch.equal(k, x) and torch.equal(v, 2 * x)


@pytest.mark.parametrize("bits8", [False, True])
def test_offsets_beyond_32_bits(bits8):
    """Pages of more than 4 GiB (and 2^32 elements of 8 bits): the last page is not the first."""
    say(f"cache of more than 2^32 bytes, 8 bits {bits8}")
    per = 8 * 64 * 128
    pages = (1 << 32) // per + 3 if bits8 else (1 << 31) // per + 3
    c = B.Pages(*(torch.empty((pages, 8, 64, 128), dtype=torch.uint8 if bits8 else BF16, device=DEV) for _ in range(2)))
    if bits8:
        c = B.Pages(c.k.view(B.E4M3), c.v.view(B.E4M3), *(torch.empty((pages, 8, 64), device=DEV) for _ in range(2)))
    table = cref.ints([[pages - 1, 0], [1, pages - 2]])
    x = torch.randn((256, 8, 128), device=DEV).to(BF16)
    start, lens = cref.starts([128, 128]), cref.ints([128, 128])
    B.cache_write(c, x, -x, start, lens, table)
    k, v = B.cache_read(c, start, table, 256, BF16)
    assert torch.equal(k, -v)
    # an 8-bit row is within half a step of e4m3 and a rounding to bfloat16
    assert bool(((k.double() - x.double()).abs() <= (x.double().abs() * (2.0 ** -4 + 2.0 ** -7) + 1e-3 if bits8 else 0.0)).all())


def test_streams_and_graphs():
    """On a stream of the caller's, and captured with the attention that reads the pages: every replay is
    the eager call, with other eager work between."""
    say("cache calls captured")
    b = cref.Cached([1, 3, 2], [40, 3, 700], 4, 2, 64, BF16, True, 16, seed=9)
    n = 6
    k, v = (torch.randn((n, 2, 64), device=DEV).to(BF16) for _ in range(2))
    pos, freq = cref.ints([39, 0, 1, 2, 698, 699]), B.rotary_frequencies(64, device=DEV)[0]

    def step():
        q, kk = B.rotate_heads(b.q, k, pos, freq)
        B.cache_write(b.cache, kk, v, b.q_start, b.k_len, b.table)
        return b.run(q=q), *B.cache_read(b.cache, cref_start, b.table, 743, BF16)

    cref_start = cref.starts([40, 3, 700])
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(step())
    for i in range(4):
        k.copy_(torch.randn_like(k))
        want = [t.clone() for t in step()]
        for graph, out in zip(graphs, outs):
            for t in out:
                t.fill_(math.nan)
            b.cache.k.view(torch.uint8)[b.table[0, 2].long(), :, 39 % 16] = 0
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, want)), f"replay {i}"
        torch.randn((1 << 20,), device=DEV).sum().item()
