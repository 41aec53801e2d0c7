"""The transformer with turned and normed heads, and over pages: chunks and single tokens as whole documents."""
from __future__ import annotations

import pytest
import torch

from paper_2401_06145_amd import binding as B
from paper_2401_06145_amd import transformer as tr
from tests import cache_ref as cref
from tests import transformer_ref as ref
from tests.gpu_helpers import DEV, say
from tests.test_gpu_transformer import ROUNDED, off, starts

pytestmark = pytest.mark.gpu

CONFIGS = [dict(), dict(rotary=32), dict(head_norm=True), dict(head_norm=True, rotary=24, factor=4.0, trained=64)]


def plain(model, x, lens, coords=None, prefix=None, causal=True):
    """The model in 64 bits, with the dequantised weights and no rounding between its steps."""
    c = model.config
    kv = c.kv_heads * c.head_dim

    def weight(w):
        q, s = w
        return q.float().double() * s.double().repeat_interleave(128, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]

    def norm(v, g):
        return ref.rms_norm(v, g, eps=c.eps)[0]

    pos = coords if coords is not None else torch.cat([torch.arange(n, device=DEV) for n in lens])
    x = x.double()
    for w in model.layers:
        q, k, v = (t.unflatten(1, (-1, c.head_dim)) for t in (norm(x, w["g_in"]) @ weight(w["qkv"]).t()).split([c.width, kv, kv], 1))
        q, k = (cref.rotate(t, pos, model.freq, w.get(g), eps=c.eps, gain=model.gain)[0] for t, g in ((q, "g_q"), (k, "g_k")))
        far = {} if coords is None else dict(slopes=model.slopes, q_pos=coords, k_pos=coords)
        o, _ = ref.attention(q, k, v, lens, lens, prefix=prefix, causal=causal, cap=c.cap, **far)
        x = x + norm(o.flatten(1), w["g_out"]) @ weight(w["out"]).t()
        x = x + norm((norm(x, w["g_up"]) @ weight(w["up"]).t()).relu(), w["g_down"]) @ weight(w["down"]).t()
    return norm(x, model.g_last)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kw", CONFIGS)
def test_whole_documents(kw, dtype):
    say(f"transformer with {kw}, whole documents, {dtype}")
    g = torch.Generator(DEV).manual_seed(1)
    lens = [150, 1, 77]
    model = tr.Transformer(tr.Config(**kw), dtype, DEV)
    x = torch.randn((sum(lens), 256), device=DEV, generator=g).to(dtype)
    got = model.forward(x, starts(lens), max(lens), causal=True)
    assert off(got, plain(model, x, lens)) < ROUNDED
    coords = torch.randint(-50, 50, (len(x), 4), device=DEV, generator=g, dtype=torch.int32)
    got = model.forward(x, starts(lens), max(lens), coords)
    assert off(got, plain(model, x, lens, coords, causal=False)) < ROUNDED


def pieces(lens):
    """New tokens of each document, call by call: prompts, chunks and single tokens, documents that wait."""
    done, calls = [0] * len(lens), []
    for sizes in ((64, 1, 0, 5), (1, 0, 150, 1), (30, 1, 70, 0), (1, 1, 1, 1)):
        new = [min(s, n - d) for s, n, d in zip(sizes, lens, done)]
        calls.append(new)
        done = [d + m for d, m in zip(done, new)]
    calls.append([n - d for n, d in zip(lens, done)])
    return calls


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("kw", CONFIGS)
def test_chunks_and_tokens(kw, bits8, dtype):
    say(f"transformer over pages with {kw}, 8 bits {bits8}, {dtype}")
    g = torch.Generator(DEV).manual_seed(2)
    lens = [120, 5, 300, 40]
    model = tr.Transformer(tr.Config(**kw), dtype, DEV)
    rows = [torch.randn((n, 256), device=DEV, generator=g).to(dtype) for n in lens]
    prefix = torch.tensor([10, 0, 40, 5], dtype=torch.int32, device=DEV) if not kw else None
    caches = model.pages(4, 40, page=16, bits8=bits8, most=20, prefix=prefix)
    out, done = [[] for _ in lens], [0] * len(lens)
    for new in pieces(lens):
        y = model.extend(torch.cat([r[d:d + m] for r, d, m in zip(rows, done, new)]), new, caches)
        at = 0
        for t, m in enumerate(new):
            out[t].append(y[at:at + m])
            at += m
            done[t] += m
    assert caches.lens == lens and caches.length.tolist() == lens
    got = torch.cat([torch.cat(o) for o in out])
    if prefix is None:  # (a prefix that arrives in chunks is seen as far as it is there)
        want = model.forward(torch.cat(rows), starts(lens), max(lens), causal=True)
        # 8-bit keys and values add the rounding of two more products
        assert off(got, want) < ROUNDED / 2 * (1.5 if bits8 else 1)
    # what the pages hold is what the first layer's product gave, turned
    k, v, start = caches.read(0)
    assert start.tolist() == starts(lens).tolist() and k.shape == (sum(lens), 2, 32) and k.dtype == dtype
    a = B.rms_norm(torch.cat(rows), model.layers[0]["g_in"], eps=model.config.eps, bits8=True)
    qkv = model._linear(a[:2], model.layers[0]["qkv"])
    wk, wv = (t.unflatten(1, (-1, 32)) for t in qkv[:, 256:].split([64, 64], 1))
    places = torch.cat([torch.arange(n, device=DEV) for n in lens])
    wk, _ = cref.rotate(wk, places, model.freq, model.layers[0].get("g_k"), eps=model.config.eps, gain=model.gain)
    # few rows and many go through products that round differently
    assert off(k, wk) < (2.0 ** -4 if bits8 else 2.0 ** -7) and off(v, wv) < (2.0 ** -4 if bits8 else 2.0 ** -7)


def test_documents_come_and_go():
    say("pages given back and out again")
    model = tr.Transformer(tr.Config(rotary=32), torch.bfloat16, DEV)
    g = torch.Generator(DEV).manual_seed(3)
    rows = torch.randn((90, 256), device=DEV, generator=g).to(torch.bfloat16)
    caches = model.pages(2, 7, page=16)
    model.extend(rows[:70], [40, 30], caches)
    caches.release(0)
    assert caches.lens == [0, 30] and len(caches.free) == 5
    again = model.extend(rows[:60], [60, 0], caches)
    alone = model.extend(rows[:60], [60], model.pages(1, 4, page=16))
    assert torch.equal(again, alone)
    with pytest.raises(ValueError):
        model.extend(rows[:80], [0, 80], caches)
    assert caches.lens == [60, 30]
    assert model.extend(rows[:0], [0, 0], caches).shape == (0, 256)
    with pytest.raises(ValueError):
        model.extend(rows[:3], [1, 1], caches)


def run_pieces(model, rows, caches, calls):
    """Outputs of each document, its calls one after the other."""
    out, done = [[] for _ in rows], [0] * len(rows)
    for new in calls:
        y = model.extend(torch.cat([r[d:d + m] for r, d, m in zip(rows, done, new)]), new, caches)
        for t, m in enumerate(new):
            out[t].append(y[sum(new[:t]):sum(new[:t + 1])])
            done[t] += m
    return torch.cat([torch.cat(o) for o in out])


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits8", [False, True])
def test_chunks_without_rotation_or_norms(bits8, dtype):
    """The base configuration: what pages and chunks alone may change."""
    say(f"transformer over pages, 8 bits {bits8}, {dtype}")
    g = torch.Generator(DEV).manual_seed(4)
    lens = [120, 5, 300, 40]
    model = tr.Transformer(tr.Config(), dtype, DEV)
    rows = [torch.randn((n, 256), device=DEV, generator=g).to(dtype) for n in lens]
    got = run_pieces(model, rows, model.pages(4, 40, page=16, bits8=bits8, most=20), pieces(lens))
    want = model.forward(torch.cat(rows), starts(lens), max(lens), causal=True)
    # 8-bit keys and values add the rounding of two more products
    assert off(got, want) < ROUNDED / 2 * (1.5 if bits8 else 1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("kw", CONFIGS)
def test_a_prefix_that_comes_in_one_call(kw, bits8, dtype):
    """Is seen by all of its document's tokens, as in whole documents."""
    say(f"transformer over pages with {kw} and a prefix, 8 bits {bits8}, {dtype}")
    g = torch.Generator(DEV).manual_seed(5)
    lens, first = [120, 5, 300, 40], [64, 5, 100, 40]
    prefix = torch.tensor([60, 0, 100, 33], dtype=torch.int32, device=DEV)
    model = tr.Transformer(tr.Config(**kw), dtype, DEV)
    rows = [torch.randn((n, 256), device=DEV, generator=g).to(dtype) for n in lens]
    caches = model.pages(4, 40, page=16, bits8=bits8, most=20, prefix=prefix)
    got = run_pieces(model, rows, caches, [first, [1, 0, 1, 0], [55, 0, 70, 0], [0, 0, 129, 0]])
    want = model.forward(torch.cat(rows), starts(lens), max(lens), causal=True, prefix=prefix)
    assert off(got, want) < ROUNDED / 2 * (1.5 if bits8 else 1)
    # and it matters: without it the first document's rows of the prefix are others
    other = model.forward(torch.cat(rows), starts(lens), max(lens), causal=True)
    assert off(want[:60], other[:60]) > 4 * ROUNDED


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("kw", CONFIGS)
def test_a_prefix_that_comes_in_chunks(kw, bits8):
    """Each call's tokens see of it what is there: one layer, whose keys go by its rows alone."""
    say(f"transformer over pages with {kw} and a prefix in chunks, 8 bits {bits8}")
    g = torch.Generator(DEV).manual_seed(6)
    n, dtype = 90, torch.bfloat16
    model = tr.Transformer(tr.Config(layers=1, **kw), dtype, DEV)
    x = torch.randn((n, 256), device=DEV, generator=g).to(dtype)
    caches = model.pages(1, 6, page=16, bits8=bits8, prefix=torch.tensor([60], dtype=torch.int32, device=DEV))
    at = 0
    for m in (20, 30, 1, 39):
        got = model.extend(x[at:at + m], [m], caches)
        at += m
        seen = torch.tensor([min(60, at)], dtype=torch.int32, device=DEV)
        want = model.forward(x[:at], starts([at]), at, causal=True, prefix=seen)[at - m:]
        assert off(got, want) < ROUNDED / 2 * (1.5 if bits8 else 1)


def test_a_refused_call_can_be_made_again():
    """Rows that the call does not take change nothing; the same tokens as they should be give what they would have given."""
    say("extend refused, and made again")
    g = torch.Generator(DEV).manual_seed(7)
    model = tr.Transformer(tr.Config(rotary=32), torch.bfloat16, DEV)
    x = torch.randn((80, 256), device=DEV, generator=g).to(torch.bfloat16)
    a, b = (model.pages(2, 9, page=16) for _ in range(2))
    for c in (a, b):
        model.extend(x[:50], [30, 20], c)
    for bad in (x[50:].float(), x[50:, :128], x[50:].clone().requires_grad_(), x[50:].cpu()):
        with pytest.raises(ValueError):
            model.extend(bad, [17, 13], a)
        assert a.lens == [30, 20] and a.length.tolist() == [30, 20] and a.free == b.free and a.held == b.held
    assert torch.equal(model.extend(x[50:], [17, 13], a), model.extend(x[50:], [17, 13], b))
    assert torch.equal(a.table[:, :2], b.table[:, :2]) and a.free == b.free
