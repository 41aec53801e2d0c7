"""The transformer over voxel features: the operators together, whole and token by token."""
from __future__ import annotations

import pytest
import torch

from paper_2401_06145_amd import net, scenes
from paper_2401_06145_amd import transformer as tr
from tests import transformer_ref as ref
from tests.gpu_helpers import DEV, say

pytestmark = pytest.mark.gpu


def starts(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEV)


def plain(model, x, lens, prefix=None, coords=None, causal=False, spacing=1):
    """The model in 64 bits, with the dequantised weights and no rounding between its steps."""
    c = model.config
    kv = c.kv_heads * c.head_dim

    def weight(w):
        q, s = w
        return q.float().double() * s.double().repeat_interleave(128, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]

    def norm(v, g):
        return ref.rms_norm(v, g, eps=c.eps)[0]

    x = x.double()
    for w in model.layers:
        q, k, v = (t.unflatten(1, (-1, c.head_dim)) for t in (norm(x, w["g_in"]) @ weight(w["qkv"]).t()).split([c.width, kv, kv], 1))
        far = {} if coords is None else dict(slopes=model.slopes / spacing, q_pos=coords, k_pos=coords)
        o, _ = ref.attention(q, k, v, lens, lens, prefix=prefix, causal=causal, cap=c.cap, **far)
        x = x + norm(o.flatten(1), w["g_out"]) @ weight(w["out"]).t()
        x = x + norm((norm(x, w["g_up"]) @ weight(w["up"]).t()).relu(), w["g_down"]) @ weight(w["down"]).t()
    return norm(x, model.g_last)


def off(got, want):
    return float((got.double() - want.double()).norm() / want.double().norm())


# A product's rows are rounded to 4 significant bits, 2^-4 / sqrt(3) of each value at most as a
# root mean square; four products a layer add to the stream, and two layers to one result.
ROUNDED = 2.0 ** -4 / 3 ** 0.5 * 4


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_whole_documents(dtype):
    say(f"transformer, whole documents, {dtype}")
    g = torch.Generator(DEV).manual_seed(1)
    lens = [150, 1, 77]
    model = tr.Transformer(tr.Config(), dtype, DEV)
    x = torch.randn((sum(lens), 256), device=DEV, generator=g).to(dtype)
    coords = 8 * torch.randint(-50, 50, (len(x), 4), device=DEV, generator=g, dtype=torch.int32)
    got = model.forward(x, starts(lens), max(lens), coords, spacing=8)
    assert got.shape == x.shape and got.dtype == dtype
    assert off(got, plain(model, x, lens, coords=coords, spacing=8)) < ROUNDED
    prefix = [60, 0, 77]
    got = model.forward(x, starts(lens), max(lens), causal=True, prefix=torch.tensor(prefix, dtype=torch.int32, device=DEV))
    assert off(got, plain(model, x, lens, prefix=prefix, causal=True)) < ROUNDED


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_token_by_token(dtype):
    """Prompts and then one token a call, as the same documents at once."""
    say(f"transformer, token by token, {dtype}")
    g = torch.Generator(DEV).manual_seed(2)
    prompts, new, room = [70, 5, 300], 6, 320
    model = tr.Transformer(tr.Config(), dtype, DEV)
    rows = [torch.randn((n + new, 256), device=DEV, generator=g).to(dtype) for n in prompts]
    prefix = torch.tensor([40, 0, 100], dtype=torch.int32, device=DEV)
    first, caches = model.prefill(torch.cat([r[:n] for r, n in zip(rows, prompts)]), starts(prompts), max(prompts), room,
                                  prefix=prefix)
    steps = [model.step(torch.stack([r[n + t] for r, n in zip(rows, prompts)]), caches) for t in range(new)]
    lens = [n + new for n in prompts]
    whole = model.forward(torch.cat(rows), starts(lens), max(lens), causal=True, prefix=prefix)
    at = 0
    for t, n in enumerate(prompts):
        mine = whole[at:at + n + new]
        at += n + new
        # different kernels round differently, which moves some 8-bit values to their neighbours
        assert off(first[sum(prompts[:t]):sum(prompts[:t + 1])], mine[:n]) < ROUNDED / 2
        assert off(torch.stack([s[t] for s in steps]), mine[n:]) < ROUNDED / 2
    assert caches.length.tolist() == lens
    with pytest.raises(ValueError):
        model.prefill(torch.cat(rows), starts(lens), max(lens), 100)
    caches.longest = room
    with pytest.raises(ValueError):
        model.step(first[:3], caches)


def test_after_a_sparse_network():
    """An encoder's voxels become the tokens; documents from their batch index."""
    say("sparse encoder, then the transformer")
    full = scenes.workload(1).coords[:20_000]
    two = torch.cat([torch.from_numpy(full), torch.from_numpy(full)]).to(DEV)
    two[len(full):, 0] += 1
    unet = net.Network(two, torch.bfloat16, ops=net.resnet_ops())
    g = torch.Generator(DEV).manual_seed(3)
    half = torch.randn((len(full), net.STEM_C), device=DEV, generator=g).to(torch.bfloat16)
    tokens = unet.forward(torch.cat([half, half]), keep=True)["s4_b1"]
    coords = unet.coords[4]
    start, longest = tr.documents(coords)
    assert start.tolist() == [0, longest, 2 * longest] and len(coords) == 2 * longest
    model = tr.Transformer(tr.Config(width=tokens.shape[1]), torch.bfloat16, DEV)
    got = model.forward(tokens, start, longest, coords, spacing=16)
    # the same scene twice: the same result twice, and the other scene plays no part
    assert torch.equal(got[:longest], got[longest:])
    alone = model.forward(tokens[:longest].contiguous(), start[:2].contiguous(), longest, coords[:longest].contiguous(),
                          spacing=16)
    assert off(alone, got[:longest]) < ROUNDED / 2
