"""spconv_cached_attention: new tokens over pages, against 64 bits and against packed keys."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests import cache_ref as cref
from tests import transformer_ref as ref
from tests.cache_ref import Cached, check_attention
from tests.gpu_helpers import DEV, say
from tests.test_gpu_cache import pages_args

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]

# queries and keys of each document, heads, key heads, columns, rows of a page
FEW = [([1], [1], 1, 1, 16, 16), ([1], [2049], 8, 2, 64, 16), ([1, 1, 1, 1], [300, 0, 17, 64], 4, 4, 32, 1),
       ([1, 5, 3], [900, 5, 4000], 8, 1, 128, 64), ([2, 1], [33, 31], 6, 2, 96, 8), ([7, 1], [500, 1], 4, 2, 256, 32),
       ([1, 1], [1500, 4097], 16, 1, 80, 2), ([4], [129], 32, 4, 128, 256)]
MANY = [([65], [65], 1, 1, 32, 16), ([130, 1, 77], [130, 300, 500], 4, 2, 64, 16), ([200], [3000], 8, 2, 128, 64),
        ([33, 0, 150], [1501, 20, 150], 12, 4, 80, 16), ([129, 64], [129, 1000], 3, 1, 96, 1), ([140, 90], [700, 91], 4, 4, 256, 32),
        ([300], [333], 2, 2, 16, 128), ([256, 70], [256, 2500], 8, 8, 48, 8)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("case", range(len(FEW) + len(MANY)))
def test_documents(case, bits8, dtype):
    ql, kl, heads, kv, d, page = (FEW + MANY)[case]
    say(f"attention over pages: {ql} of {kl}, {heads} heads on {kv} of {d}, pages of {page}, 8 bits {bits8}, {dtype}")
    b = Cached(ql, kl, heads, kv, d, dtype, bits8, page, seed=case)
    slopes = torch.exp2(-torch.arange(heads, device=DEV) / 2)
    for kw in (dict(), dict(causal=False), dict(cap=20.0), dict(slopes=slopes), dict(cap=70.0, slopes=slopes, scale=0.3),
               dict(prefix=[n // 2 for n in kl])):
        got = b.run(**kw)
        assert got.shape == b.q.shape and got.dtype == dtype
        want, mag = b.want(**kw)
        check_attention(got, want, mag, str(kw.keys()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", [1, 3, 9, 10, 12])
def test_as_over_packed_keys(case, dtype):
    """The same keys packed: the same kernels but for where a row comes from, and the same bits; float32 rows of
    more than 64 columns go through tiles of half the keys, so that sums have another order."""
    ql, kl, heads, kv, d, page = (FEW + MANY)[case]
    say(f"attention over pages and packed keys {ql} of {kl} {dtype}")
    b = Cached(ql, kl, heads, kv, d, dtype, False, page, seed=case)
    packed = B.attention(b.q, b.k.to(dtype), b.v.to(dtype), b.q_start, cref.starts(kl), max(ql), max(kl), causal=True)
    if dtype != F32 or d <= 64:
        assert torch.equal(b.run(), packed)
    else:
        check_attention(b.run(), packed.double(), b.want()[1], "pages and packed keys")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits8", [False, True])
def test_rows_that_see_nothing(bits8, dtype):
    """More queries than keys: the first see none, and get zeros; so do those of an empty document."""
    say(f"queries before the first key, 8 bits {bits8} {dtype}")
    for ql, kl in (([9, 4, 3], [4, 0, 3]), ([200, 130, 70], [30, 0, 1])):
        b = Cached(ql, kl, 4, 2, 64, dtype, bits8, 8, seed=3)
        got = b.run()
        want, mag = b.want()
        check_attention(got, want, mag, "causal")
        assert bool((got[:ql[0] - kl[0]] == 0).all()) and bool((got[ql[0]:ql[0] + ql[1]] == 0).all())
        check_attention(b.run(prefix=[2, 5, 0]), *b.want(prefix=[2, 5, 0]), "with a prefix")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("ql,kl", [([3, 5], [40, 300]), ([150, 70], [200, 900])])
def test_hidden_keys_may_hold_anything(ql, kl, bits8, dtype):
    """A key that a query does not see adds nothing to it, whatever its values; those that see it get them."""
    say(f"NaN and infinities among hidden values {ql} of {kl}, 8 bits {bits8} {dtype}")
    heads, kv, d = 4, 2, 64
    plain = Cached(ql, kl, heads, kv, d, dtype, bits8, 16, seed=5)
    for value in (math.nan, math.inf, -math.inf):
        k, v = (torch.randn((sum(kl), kv, d), device=DEV) for _ in range(2))
        v[kl[0] - 2, :, 3] = value                 # seen by the last two queries of document 0
        v[sum(kl) - 1, 1, 9] = value               # by the last of document 1, in one head
        b = Cached(ql, kl, heads, kv, d, dtype, bits8, 16, seed=5, like=(k, v))
        clean = Cached(ql, kl, heads, kv, d, dtype, bits8, 16, seed=5,
                       like=(k, torch.where(v.isfinite(), v, 0.0)))
        got, want = b.run(), clean.run()
        sees = torch.zeros(b.q.shape, dtype=torch.bool, device=DEV)
        # the scale of such a row of 8 bits is infinite, or (by torch's maximum) NaN: the whole row is NaN
        whole = bits8
        sees[ql[0] - 2:ql[0], :, slice(None) if whole else 3] = True
        sees[sum(ql) - 1, heads // 2:, slice(None) if whole else 9] = True
        assert not bool(got[sees].isfinite().any())
        if not bits8:  # (the rows' scales differ with the value)
            mag = clean.want()[1]
            off = (got.double() - want.double()).abs()
            u = ref.UNIT[dtype]
            assert bool((off[~sees] <= (mag * (2 * u + 4e-5) + u * want.double().abs())[~sees]).all())
        assert bool(got[~sees].isfinite().all())
    assert bool(plain.run().isfinite().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ql,kl", [([3, 5], [40, 300]), ([150, 70], [200, 900])])
def test_hidden_nan_of_8_bits(ql, kl, dtype):
    """A NaN that cache_write has put into a row of 8 bits, whose scale stays finite, is one column's."""
    say(f"one NaN in a row of 8 bits {ql} of {kl} {dtype}")
    b = Cached(ql, kl, 4, 2, 64, dtype, True, 16, seed=15)
    want, mag = b.want()
    last = [torch.randn((2, 2, 64), device=DEV).to(dtype) for _ in range(2)]  # a new last key of each document
    B.cache_write(b.cache, *last, cref.starts([1, 1]), b.k_len, b.table)
    clean = b.run()
    last[1][1, 1, 9] = math.nan
    last[1][1, 1, 8] = last[1][1, 1].nan_to_num(0.0).abs().max() * 1.5  # the largest, in both
    B.cache_write(b.cache, *last, cref.starts([1, 1]), b.k_len, b.table)
    got = b.run()
    sees = torch.zeros(b.q.shape, dtype=torch.bool, device=DEV)
    sees[sum(ql) - 1, 2:, 9] = True
    assert bool(got[sees].isnan().all()) and bool(got[~sees].isfinite().all())
    # queries that do not see it are as before
    assert torch.equal(got[:-1], clean[:-1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e-4, 1.0, 1e4, 1e30])
def test_scales_of_all_sizes(size, dtype):
    """8-bit values far from 1, and rows of very different scales side by side."""
    if dtype == F16 and size not in (1e-4, 1.0, 1e4):
        return  # float16 has no such values
    say(f"8-bit values of {size} {dtype}")
    for ql, kl, d in (([1, 3], [700, 90], 64), ([150], [333], 128)):
        k, v = (torch.randn((sum(kl), 2, d), device=DEV) for _ in range(2))
        mixed = torch.exp2(torch.randint(-6, 1, (sum(kl), 2, 1), device=DEV).float())
        for spread in (torch.ones_like(mixed), mixed):
            b = Cached(ql, kl, 4, 2, d, dtype, True, 16, seed=6, like=(k * spread, v * size * spread))
            want, mag = b.want()
            u = ref.UNIT[dtype]
            # float16: each value may be rounded to a subnormal (2^-25)
            bound = mag * (2 * u + 4e-5) + want.abs() * u + 2 * ref.TINY[dtype]
            off = (b.run().double() - want).abs()
            assert bool((off <= bound).all()), f"{float((off / bound).max()):.2f} of the bound"


def test_weak_keys_beside_a_dominant_one():
    """float16: many keys whose exponentials are small keep their part of the sum, also with small scales."""
    say("weak keys in float16")
    n, d = 8192, 64
    k = torch.zeros((n, 1, d), device=DEV)
    v = torch.ones((n, 1, d), device=DEV)
    k[5, 0, 0] = 8.0
    v[5] = 0.0
    for size in (1.0, 0.007):
        for ql in ([1], [100]):
            b = Cached(ql, [n], 1, 1, d, F16, True, 64, seed=7, like=(k, v * size))
            b.q[:] = 0.0
            b.q[..., 0] = 2.0  # 16 beside 0: e^-16 each, 8191 of them
            kw = dict(scale=1.0, causal=False)
            check_attention(b.run(**kw), *b.want(**kw), f"values of {size}")


@pytest.mark.parametrize("bits8", [False, True])
def test_pages_that_are_none(bits8):
    """A table entry outside the pages stands for zeros, and is never followed."""
    say(f"attention over missing pages, 8 bits {bits8}")
    for ql, kl in (([1, 2], [300, 40]), ([150, 90], [300, 100])):
        for wrong in (-1, -(1 << 31), (1 << 31) - 1, None):
            b = Cached(ql, kl, 4, 2, 64, BF16, bits8, 16, seed=8)
            b.table[0, 3], b.table[1, 1] = (wrong if wrong is not None else len(b.cache.k),) * 2
            for t, first in ((0, 48), (1, kl[0] + 16)):
                b.k[first:first + 16] = 0.0
                b.v[first:first + 16] = 0.0
            check_attention(b.run(), *b.want(), f"entry {wrong}")


def test_shared_pages_and_repeats():
    """Documents that share their first pages; the same bits in every call."""
    say("shared pages")
    for ql, kl in (([1, 1, 1], [500, 500, 500]), ([70, 70, 70], [500, 500, 500])):
        b = Cached(ql, kl, 8, 2, 64, BF16, True, 16, seed=9)
        b.table[1, :20] = b.table[0, :20]
        b.k[500:820], b.v[500:820] = b.k[:320], b.v[:320]
        got = b.run()
        check_attention(got, *b.want(), "shared")
        assert all(torch.equal(b.run(), got) for _ in range(3))


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("ql,kl", [([4, 3, 2], [4000, 30, 900]), ([300, 100, 70], [900, 100, 700])])
def test_rows_without_output_stay_as_they_are(ql, kl, bits8):
    """Rows before the first document and behind the last, and queries behind max_q."""
    say(f"attention over pages with rows of no document {ql} of {kl}, 8 bits {bits8}")
    before, behind, heads, kv, d = 5, 130, 8, 2, 64
    b = Cached(ql, kl, heads, kv, d, F16, bits8, 16, seed=10)
    want, mag = b.want()
    q = torch.cat([torch.full((before, heads, d), math.nan, device=DEV).to(F16), b.q,
                   torch.full((behind, heads, d), math.nan, device=DEV).to(F16)])
    start = b.q_start + before
    p = pages_args(b.cache, b.table)
    for max_q in (max(ql), max(1, max(ql) // 2)):
        out = torch.full_like(q, 7.0)
        a = B.AttentionArgs(d_q=q.data_ptr(), d_out=out.data_ptr(), q_row=heads * d, q_head=d, out_row=heads * d, out_head=d,
                            d_q_start=start.data_ptr(), d_k_len=b.k_len.data_ptr(), n_q=len(q), n_docs=len(ql), max_q=max_q,
                            max_k=max(kl), heads=heads, kv_heads=kv, head_dim=d, dtype=B.SPCONV_F16, causal=1, scale=d ** -0.5)
        need = B.spconv_cached_attention_workspace_bytes(p, a)
        ws = torch.full((need // 4,), math.nan, device=DEV).view(torch.uint8) if need else None
        B.spconv_cached_attention(p, a, ws)
        has = torch.zeros(len(q), dtype=torch.bool, device=DEV)
        for t, n in enumerate(ql):
            at = before + sum(ql[:t])
            has[at:at + min(n, max_q)] = True
        assert bool((out[~has] == 7).all())
        if max_q == max(ql):
            check_attention(out[has], want, mag, "the documents")


def test_offsets_beyond_32_bits():
    """Keys in the first and the last pages of a cache of more than 4 GiB."""
    say("attention over more than 2^32 bytes of pages")
    for bits8 in (False, True):
        per = 8 * 64 * 128
        pages = (1 << 32) // per + 3 if bits8 else (1 << 31) // per + 3
        shape = (pages, 8, 64, 128)
        c = B.Pages(*(torch.empty(shape, dtype=torch.uint8, device=DEV).view(B.E4M3) if bits8
                      else torch.empty(shape, dtype=BF16, device=DEV) for _ in range(2)))
        if bits8:
            c.k_scale, c.v_scale = (torch.empty(shape[:3], device=DEV) for _ in range(2))
        small = {}
        for ql in ([1, 1], [100, 64]):
            b = Cached(ql, [200, 128], 8, 8, 128, BF16, bits8, 64, seed=11)
            big = cref.ints([[pages - 1, 0, pages - 3, 2], [1, pages - 2, 5, 5]])
            for t, m in ((0, 4), (1, 2)):
                for name in ("k", "v", "k_scale", "v_scale"):
                    if getattr(c, name) is not None:
                        to, of = getattr(c, name), getattr(b.cache, name)
                        view = (lambda x: x.view(torch.uint8)) if name in "kv" and bits8 else (lambda x: x)
                        view(to)[big[t, :m].long()] = view(of)[b.table[t, :m].long()]
            got = b.run(cache=c, table=big)
            assert torch.equal(got, b.run())
            small[len(ql)] = got
        del c


def test_no_queries_no_documents_no_pages():
    say("empty calls")
    b = Cached([2, 1], [0, 0], 4, 2, 64, F16, False, 16, spare=0)
    assert b.cache.k.shape[0] == 0 and bool((b.run(max_k=5) == 0).all())
    b8 = Cached([2, 1], [0, 0], 4, 2, 64, F16, True, 16, spare=0)
    assert bool((b8.run(max_k=5) == 0).all())
    none = Cached([], [], 4, 2, 64, F16)
    assert none.run(max_q=1, max_k=1).shape == (0, 4, 64)


def test_strided_queries():
    """A slice of a fused product."""
    say("attention over pages, strided queries")
    b = Cached([3, 60], [100, 70], 4, 2, 64, BF16, True, 16, seed=12)
    wide = torch.randn((63, 8, 64), device=DEV).to(BF16)
    wide[:, 2:6] = b.q
    assert torch.equal(b.run(q=wide[:, 2:6]), b.run())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits8", [False, True])
def test_slopes_of_all_sizes(bits8, dtype):
    """A bias by place of any size, also far from the queries."""
    say(f"slopes of all sizes over pages, 8 bits {bits8} {dtype}")
    for ql, kl in (([3, 1], [700, 90]), ([150, 70], [200, 3000])):
        b = Cached(ql, kl, 8, 2, 64, dtype, bits8, 32, seed=13)
        slopes = torch.tensor([0.0, 1e-6, 1e-3, 1.0, -1e-2, 1e20, 1e37, math.inf], device=DEV)
        got = b.run(slopes=slopes)
        assert bool(got[:, 7].isnan().all())  # infinity times the distance 0
        want, mag = b.want(slopes=slopes)
        check_attention(got[:, :7], want[:, :7], mag[:, :7], "finite slopes")
        for causal, prefix in ((False, None), (True, [n // 2 for n in kl])):
            got = b.run(slopes=slopes[:7].repeat(2)[:8].contiguous(), causal=causal, prefix=prefix)
            want, mag = b.want(slopes=slopes[:7].repeat(2)[:8], causal=causal, prefix=prefix)
            check_attention(got, want, mag, f"causal {causal}, prefix {prefix}")


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [1, 2, 4, 8, 16, 32, 64, 128, 1024])
def test_pages_of_all_sizes(page, bits8):
    """Pages that end inside a tile, hold many tiles, or one row; every width."""
    say(f"attention over pages of {page}, 8 bits {bits8}")
    for d in (16, 32, 64, 96, 128, 256):
        for ql, kl, dtype in (([70, 1, 200], [77, 300, 517], BF16), ([1, 2], [517, 64], F32), ([65], [129], F32)):
            b = Cached(ql, kl, 2, 1, d, dtype, bits8, page, seed=page + d)
            check_attention(b.run(), *b.want(), f"{d} columns, {ql} of {kl}, {dtype}")
            check_attention(b.run(cap=15.0, prefix=[n // 3 for n in kl]), *b.want(cap=15.0, prefix=[n // 3 for n in kl]), "capped")


def test_lengths_at_the_ends_of_tiles():
    """Every length around the ends of pages, tiles and ranges."""
    say("attention over pages, lengths from 1 to 260")
    for ql in (1, 40):
        for dtype, bits8 in ((BF16, True), (F16, False), (F32, True)):
            kl = [n for n in range(1, 261) if min(n % 16, -n % 16) <= 1]
            b = Cached([min(ql, n) for n in kl], kl, 4, 2, 32, dtype, bits8, 16, seed=14)
            check_attention(b.run(), *b.want(), f"{ql} queries {dtype}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("size", [1e4, 1e9, 1e14])
def test_scores_of_all_sizes(size, bits8, dtype):
    """Scores far beyond what exponentials take: the largest wins, wherever it is, whatever its sign."""
    say(f"scores of {size} over pages, 8 bits {bits8} {dtype}")
    for ql, kl in (([3, 1], [700, 90]), ([150], [400])):
        b = Cached(ql, kl, 4, 2, 64, dtype, bits8, 32, seed=16)
        towards = torch.sign(torch.randn(64, device=DEV))
        for sign in (1.0, -1.0):
            # keys i (2 + i) / 1024 along one direction, apart by more than any rounding of the scores
            k = torch.cat([(2 + torch.arange(n, device=DEV).flip(0)) / 1024 for n in kl])[:, None, None] * towards
            c = Cached(ql, kl, 4, 2, 64, dtype, bits8, 32, seed=16, like=(k.expand(-1, 2, -1).contiguous(), torch.randn((sum(kl), 2, 64), device=DEV)))
            c.q[:] = (sign * size * towards).to(dtype)
            got, (want, mag) = c.run(scale=1.0, causal=False), c.want(scale=1.0, causal=False)
            # 8-bit keys share values, 16-bit ones some: where two largest are equal both count
            check_attention(got, want, mag, f"{sign}")
