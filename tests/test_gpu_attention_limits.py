"""spconv_attention at the ends of what it accepts: caps, strides, rows outside of the call's
documents, values and lengths far from the ordinary."""
from __future__ import annotations

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests import transformer_ref as ref
from tests.gpu_helpers import DEV, say
from tests.test_gpu_attention import Batch, ints

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap", [1e-40, 1e-3, 0.5, 64.0, 65.0, 200.0, 1e3, 1e4, 1e6, 1e12, 1e30])
def test_caps_of_all_sizes(cap, dtype):
    """A cap far above the scores leaves them as they are: its error must not grow with the cap."""
    say(f"attention with a cap of {cap} {dtype}")
    for ql, kl, d in (([150, 40], [150, 333], 64), ([1, 3], [700, 90], 128), ([130], [200], 256)):
        for spread in (1.0, 12.0, 100.0):
            b = Batch(ql, kl, 4, 2, d, dtype, spread=spread, seed=21)
            for bias in ("none", "position", "voxel"):
                got = b.run(causal=True, cap=cap, bias=bias)
                want, mag = ref.attention(b.q, b.k, b.v, b.q_lens, b.k_lens, causal=True, cap=cap, **b.bias(bias))
                u = ref.UNIT[dtype]  # float32 errors of the scores grow with them, and end at the cap
                bound = mag * (2 * u + 4e-5 * max(1.0, min(spread, cap))) + want.abs() * u + ref.TINY[dtype]
                off = (got.double() - want).abs()
                assert bool((off <= bound).all()), f"{bias}, scores of {spread}: {float((off / bound).max()):.2f} of the bound"


SET_BEFORE = 7.0


def run_into(b, q_start, k_start, max_q, max_k, causal=True):
    """The C call on an output that is set before and a workspace of NaN: (output, bytes of workspace)."""
    heads, kv, d, n, nk = b.q.shape[1], b.k.shape[1], b.q.shape[2], len(b.q), len(b.k)
    out = torch.full_like(b.q, SET_BEFORE)
    qs, ks = ints(q_start), ints(k_start)
    a = B.AttentionArgs(d_q=b.q.data_ptr(), d_k=b.k.data_ptr(), d_v=b.v.data_ptr(), d_out=out.data_ptr(),
                        q_row=heads * d, q_head=d, k_row=kv * d, k_head=d, v_row=kv * d, v_head=d, out_row=heads * d, out_head=d,
                        d_q_start=qs.data_ptr(), d_k_start=ks.data_ptr(), n_q=n, n_k=nk, n_docs=len(q_start) - 1,
                        max_q=max_q, max_k=max_k, heads=heads, kv_heads=kv, head_dim=d, dtype=B.DTYPES[b.q.dtype],
                        causal=causal, scale=d ** -0.5)
    need = B.spconv_attention_workspace_bytes(a)
    workspace = torch.full((need // 4,), float("nan"), device=DEV).view(torch.uint8) if need else None
    B.spconv_attention(a, workspace)
    torch.cuda.synchronize()
    return out, need


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_documents_from_the_middle_of_a_batch(dtype):
    """A call on the documents from t on leaves the rows of those before as they are."""
    say(f"attention on the last documents of a batch {dtype}")
    for ql, kl, heads in (([300, 100, 70], [64, 60, 64], 2), ([127, 1, 200], [30, 64, 64], 1), ([5000, 64, 130], [9, 60, 64], 2)):
        b = Batch(ql, kl, heads, heads, 32, dtype, seed=31)
        want, mag = ref.attention(b.q, b.k, b.v, ql, kl, causal=True)
        for t in (1, 2):
            at = [sum(ql[:i]) for i in range(t, len(ql) + 1)]
            got, need = run_into(b, at, [sum(kl[:i]) for i in range(t, len(kl) + 1)], max(ql[t:]), 64)
            assert need == 0
            assert bool((got[:at[0]] == SET_BEFORE).all()), f"rows before {at[0]}"
            ref.check_attention(got[at[0]:], want[at[0]:], mag[at[0]:], f"documents from {t} on")


# queries and keys of each document, heads, key heads, width, whether the keys are split: few queries and many
GAPS = [([4, 3, 2], [40, 30, 20], 8, 2, 64, False), ([4, 3, 2], [4000, 30, 900], 8, 2, 64, True),
        ([1, 1, 1], [9000, 20, 12_000], 4, 1, 128, True), ([300, 100, 70], [64, 64, 64], 2, 2, 32, False),
        ([300, 100, 70], [900, 100, 700], 2, 2, 32, True), ([130, 1, 200], [6000, 1, 3000], 1, 1, 256, True)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("case", range(len(GAPS)))
def test_rows_without_output_stay_as_they_are(case, dtype):
    """Rows before the first document and behind the last (a batch padded to a fixed number of
    rows), and queries behind max_q, whether the keys are split into ranges or not."""
    ql, kl, heads, kv, d, split = GAPS[case]
    say(f"attention with rows of no document, {ql} queries, {kl} keys, {d} columns, {dtype}")
    before, behind = 5, 130
    lens = [before, *ql, behind]
    b = Batch(lens, [0, *kl, 0], heads, kv, d, dtype, seed=41)
    at = [sum(lens[:i]) for i in range(1, len(lens))]
    k_at = [sum(kl[:i]) for i in range(len(kl) + 1)]
    want, mag = ref.attention(b.q, b.k, b.v, lens, [0, *kl, 0], causal=True)
    for max_q in (max(ql), max(1, max(ql) - 1), max(1, max(ql) // 2)):
        got, need = run_into(b, at, k_at, max_q, max(kl))
        assert (need > 0) == split
        has = torch.zeros(len(b.q), dtype=torch.bool, device=DEV)
        for t, n in enumerate(ql):
            has[at[t]:at[t] + min(n, max_q)] = True
        assert bool((got[~has] == SET_BEFORE).all()), f"max_q {max_q}"
        if max_q == max(ql):
            ref.check_attention(got[has], want[has], mag[has], "the documents")
        else:
            assert bool(got[has].isfinite().all()) and not bool((got[has] == SET_BEFORE).all())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap", [20.0, 50.0, 60.0])
@pytest.mark.parametrize("size", [1e-30, 1e-20, 1.0, 1e20, 1e33])
def test_large_and_small_values_of_capped_keys(size, cap, dtype):
    """Whatever the scores (all near -cap, all near +cap, small ones, one after the other), values
    of every size keep it: exponentials are relative to the largest."""
    if dtype == F16 and size != 1.0:
        return  # float16 has no such values
    say(f"attention with values of {size} under a cap of {cap} {dtype}")
    for ql, kl, d in (([150, 40], [150, 333], 64), ([200], [700], 128), ([3, 1], [700, 90], 64)):
        b = Batch(ql, kl, 4, 2, d, dtype, seed=51)
        b.v = (b.v.float() * size).to(dtype)
        towards = torch.randn(d, device=DEV)
        for near in (1.0, -1.0, 0.0, 0.02):
            # keys along one direction; queries along it, against it, small, or each differently
            b.k = (torch.randn(b.k.shape, device=DEV) * 0.1 + towards).to(dtype)
            q = torch.randn(b.q.shape, device=DEV) * 0.1 + (30 * near) * towards
            if near == 0.02:
                q *= torch.exp2(torch.randint(-3, 6, q.shape[:2], device=DEV).float())[..., None]
            b.q = q.to(dtype)
            got = b.run(causal=True, cap=cap)
            want, mag = ref.attention(b.q, b.k, b.v, ql, kl, causal=True, cap=cap)
            u = ref.UNIT[dtype]
            # float32 errors of scores of up to the cap, products of up to some hundred behind them
            bound = mag * (2 * u + 4e-5 * 30) + want.abs() * u + ref.TINY[dtype]
            off = (got.double() - want).abs()
            assert bool((off <= bound).all()), f"{near}: {float((off / bound).max()):.2f} of the bound"


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_infinite_products_under_a_cap(dtype):
    """A product of -inf is a score of -cap, one of +inf a score of cap."""
    say(f"attention with infinite products under a cap {dtype}")
    for ql, kl, d in (([150, 40], [150, 333], 64), ([200], [700], 128), ([3, 1], [700, 90], 64)):
        for first, last in ((0, 64), (0, 90), (10, 70), (40, 41)):
            for sign in (-1.0, 1.0):
                b = Batch(ql, kl, 4, 2, d, dtype, seed=61)
                b.q = b.q.abs()
                b.k[first:last] = sign * float("inf")
                got = b.run(causal=True, cap=20.0)
                want, mag = ref.attention(b.q, b.k, b.v, ql, kl, causal=True, cap=20.0)
                ref.check_attention(got, want, mag, f"keys {first} to {last}, {sign}")


@pytest.mark.parametrize("dtype", [F32, F16])
@pytest.mark.parametrize("d,stride", [(8, 32 << 20), (24, 17 << 20), (24, 32 << 20), (40, 24 << 20), (64, 32 << 20)])
def test_keys_far_apart(d, stride, dtype):
    """Rows of keys and values up to 32 MiB apart, everything between them NaN: 128 of them span 4 GiB."""
    say(f"attention with rows of {d} columns {stride} bytes apart {dtype}")
    n, e = 140, torch.empty((), dtype=dtype).element_size()
    b = Batch([n], [n], 2, 1, d, dtype, seed=71)
    wide = torch.full((n, stride // e), float("nan"), device=DEV, dtype=dtype)
    k, v = wide[:, :d].unflatten(1, (1, d)), wide[:, 2 * d:3 * d].unflatten(1, (1, d))
    k.copy_(b.k), v.copy_(b.v)
    s = ints([0, n])
    for bias in ("none", "voxel"):
        want, mag = ref.attention(b.q, b.k, b.v, [n], [n], **b.bias(bias))
        ref.check_attention(B.attention(b.q, k, v, s, s, n, n, **b.bias(bias)), want, mag, bias)
        few = torch.tensor([0, 5], dtype=torch.int32, device=DEV)
        got = B.attention(b.q[:5], k, v, few, s, 5, n, **{**b.bias(bias), **({"q_pos": b.q_pos[:5]} if bias == "voxel" else {})})
        ref.check_attention(got, want[:5], mag[:5], f"few queries, {bias}")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("below", [12.0, 25.6, 30.0])
def test_many_weak_keys_beside_a_dominant_one(below, dtype):
    """Keys whose weights are 2^-below of the largest keep their part of a long document's result."""
    say(f"attention with weights of 2^-{below} {dtype}")
    n, d, heads = 100_000, 64, 2
    g = torch.Generator(DEV).manual_seed(81)
    for ql in (1, 130):
        q = torch.zeros((ql, heads, d), device=DEV)
        k = torch.zeros((n, heads, d), device=DEV)
        q[..., 0], k[..., 0] = 16.0, (32.0 - below * 0.6931472) / 2.0
        k[n // 3, :, 0] = 16.0
        k[..., 1] = torch.randn((n, heads), device=DEV, generator=g)  # not seen by the queries
        v = 1.0 + 0.1 * torch.randn((n, heads, d), device=DEV, generator=g)
        v[n // 3] = 0.0
        q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
        pos = torch.randint(0, 50, (n, 4), device=DEV, generator=g, dtype=torch.int32)
        slopes = torch.full((heads,), 1e-6, device=DEV)
        for bias in ({}, dict(slopes=slopes), dict(slopes=slopes, q_pos=pos[:ql], k_pos=pos)):
            got = B.attention(q, k, v, ints([0, ql]), ints([0, n]), ql, n, **bias)
            want, mag = ref.attention(q, k, v, [ql], [n], **bias)
            ref.check_attention(got, want, mag, f"{ql} queries")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_near_places_of_a_document_of_more_than_2_24_keys(dtype):
    """Distances of one or two count, wherever in the document."""
    n, d, tail = (1 << 24) + 1001, 8, 600
    say(f"attention with a bias by place over {n} keys {dtype}")
    g = torch.Generator(DEV).manual_seed(91)
    k, v = (torch.zeros((n, 1, d), device=DEV, dtype=dtype) for _ in range(2))
    k[-tail:], v[-tail:] = (torch.randn((tail, 1, d), device=DEV, generator=g).to(dtype) for _ in range(2))
    slopes = torch.tensor([1.0], device=DEV)
    for ql in (1, 5, 130):
        q = torch.randn((ql, 1, d), device=DEV, generator=g).to(dtype)
        got = B.attention(q, k, v, ints([0, ql]), ints([0, n]), ql, n, causal=True, slopes=slopes)
        # keys 400 places and more before a query weigh e^-400
        want, mag = ref.attention(q, k[-tail:].contiguous(), v[-tail:].contiguous(), [ql], [tail], causal=True, slopes=slopes)
        ref.check_attention(got, want, mag, f"{ql} queries")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_slopes_up_to_the_largest_number(dtype):
    """A slope of float32's largest number leaves the key at distance 0 alone."""
    say(f"attention with the steepest slopes {dtype}")
    for ql, d in (([150], 64), ([3], 128)):
        b = Batch(ql, ql, 2, 2, d, dtype, seed=101)
        b.k_pos = b.q_pos = torch.arange(ql[0] * 4, device=DEV, dtype=torch.int32).view(-1, 4)
        slopes = torch.tensor([3.4028234e38, 1e38], device=DEV)
        for bias in (dict(slopes=slopes), dict(slopes=slopes, q_pos=b.q_pos, k_pos=b.k_pos)):
            for cap in (0.0, 20.0):
                want, mag = ref.attention(b.q, b.k, b.v, ql, ql, causal=True, cap=cap, **bias)
                assert torch.equal(want, b.v.double())
                ref.check_attention(b.run(causal=True, cap=cap, bias="none", **bias), want, mag, "steepest slopes")
