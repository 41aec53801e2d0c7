"""A transformer over voxel features, built from the library's operators: what follows a sparse
network whose voxels become the tokens of scenes (a batch's scenes are the documents).

One layer (every product reads 8-bit rows that a norm has written; sums of the residual stream
are part of the norms):

  a    = norm(x + what the layer before added)          spconv_rms_norm, e4m3 and scales
  qkv  = a Wqkv                                          spconv_scaled_linear
  o    = attention(q, k, v) inside each scene            spconv_attention
  x   += norm(o) Wout
  u    = relu(norm(x) Wup)
  x   += norm(u) Wdown

``forward`` runs whole documents: voxels that all see each other, nearer ones counting more
(``causal=False`` with coordinates), or a scene's tokens as a prefix that all see, with text after
it that sees backwards.  ``prefill`` and ``step`` are the same with caches: a batch's prompts, then
one new token for each document a call.

    python -m paper_2401_06145_amd.transformer      # a small UNet encoder, its voxels, ten new tokens
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as B


@dataclass
class Config:
    width: int = 256
    heads: int = 8
    kv_heads: int = 2
    layers: int = 2
    inner: int = 1024
    cap: float = 30.0     # of the scores; 0: none
    eps: float = 1e-6
    exact: bool = False   # products summed in float32 throughout (spconv_scaled_linear's exact), at about half the rate

    @property
    def head_dim(self) -> int:
        return self.width // self.heads


@dataclass
class Caches:
    """Keys and values of each layer: ``room`` rows for each document, ``length`` of them filled."""
    k: list
    v: list
    start: torch.Tensor    # int32 [docs + 1], multiples of room
    length: torch.Tensor   # int32 [docs]
    prefix: torch.Tensor | None
    room: int
    longest: int           # the longest length, known to the host


def documents(coords: torch.Tensor) -> tuple[torch.Tensor, int]:
    """(first row of each scene, longest scene) of coordinates sorted by batch index, as every
    downsampled level's are: int32 [scenes + 1] for ``forward``, and a length for the host."""
    batch = coords[:, 0].contiguous()
    scenes = int(batch[-1]) + 1 if len(batch) else 0
    start = torch.searchsorted(batch, torch.arange(scenes + 1, device=coords.device, dtype=batch.dtype)).to(torch.int32)
    return start, int((start[1:] - start[:-1]).max()) if scenes else 0


class Transformer:
    """Weights of one model (random, from a seed), quantised once."""

    def __init__(self, config: Config, dtype: torch.dtype = torch.bfloat16, device="cuda", seed: int = 50_000):
        self.config, self.dtype, self.device = config, dtype, torch.device(device)
        c = config
        g = torch.Generator(device="cpu").manual_seed(seed)

        def weight(n, k):
            return B.quantize_weight((torch.randn((n, k), generator=g) / k ** 0.5).to(self.device))

        def gamma(n):
            return (1 + 0.1 * torch.randn(n, generator=g)).to(self.device, dtype)

        kv = c.kv_heads * c.head_dim
        self.layers = [dict(qkv=weight(c.width + 2 * kv, c.width), out=weight(c.width, c.width),
                            up=weight(c.inner, c.width), down=weight(c.width, c.inner), g_in=gamma(c.width),
                            g_out=gamma(c.width), g_up=gamma(c.width), g_down=gamma(c.inner)) for _ in range(c.layers)]
        self.g_last = gamma(c.width)
        self.slopes = torch.exp2(-8.0 * torch.arange(1, c.heads + 1) / c.heads).to(self.device)

    def _linear(self, rows, weight, relu=False):
        return B.scaled_linear(rows[0], rows[1], weight[0], weight[1], self.dtype, relu=relu, exact=self.config.exact)

    def _run(self, x: torch.Tensor, attend) -> torch.Tensor:
        """The layers on rows x; attend(layer, q, k, v) is their attention."""
        c = self.config
        kv = c.kv_heads * c.head_dim
        add = None
        for i, w in enumerate(self.layers):
            *a, total = B.rms_norm(x, w["g_in"], residual=add, eps=c.eps, bits8=True)
            x = x if add is None else total
            q, k, v = (t.unflatten(1, (-1, c.head_dim)) for t in self._linear(a, w["qkv"]).split([c.width, kv, kv], 1))
            o = attend(i, q, k, v).flatten(1)
            add = self._linear(B.rms_norm(o, w["g_out"], eps=c.eps, bits8=True)[:2], w["out"])
            *a, x = B.rms_norm(x, w["g_up"], residual=add, eps=c.eps, bits8=True)
            u = self._linear(a, w["up"], relu=True)
            add = self._linear(B.rms_norm(u, w["g_down"], eps=c.eps, bits8=True)[:2], w["down"])
        return B.rms_norm(x, self.g_last, residual=add, eps=c.eps)[0]

    def forward(self, x: torch.Tensor, start: torch.Tensor, longest: int, coords: torch.Tensor | None = None,
                causal: bool = False, prefix: torch.Tensor | None = None, spacing: int = 1) -> torch.Tensor:
        """Whole documents: rows x [n][width], document t being rows start[t] .. start[t + 1].  With
        coords, scores fall with the voxels' distance, in units of ``spacing`` (the level's)."""
        slopes = None if coords is None else self.slopes / spacing
        return self._run(x, lambda i, q, k, v: B.attention(
            q, k, v, start, start, longest, longest, prefix=prefix, causal=causal, cap=self.config.cap, slopes=slopes,
            q_pos=coords, k_pos=coords))

    def prefill(self, x: torch.Tensor, start: torch.Tensor, longest: int, room: int,
                prefix: torch.Tensor | None = None) -> tuple[torch.Tensor, Caches]:
        """Prompts (causal, with an optional prefix that all see), and caches of ``room`` keys a document."""
        c, docs = self.config, len(start) - 1
        if longest > room:
            raise ValueError(f"a prompt of {longest} tokens does not fit caches of {room}")
        length = start[1:] - start[:-1]
        row = torch.arange(len(x), device=self.device)
        doc = torch.searchsorted(start[1:].contiguous(), row, right=True)
        at = doc * room + row - start[doc]
        shape = (docs * room, c.kv_heads, c.head_dim)
        caches = Caches([], [], torch.arange(docs + 1, device=self.device, dtype=torch.int32) * room, length.contiguous(),
                        prefix, room, longest)

        def attend(i, q, k, v):
            for kept, new in ((caches.k, k), (caches.v, v)):
                kept.append(torch.empty(shape, dtype=self.dtype, device=self.device))
                kept[-1][at] = new
            return B.attention(q, k, v, start, start, longest, longest, prefix=prefix, causal=True, cap=c.cap)

        return self._run(x, attend), caches

    def step(self, x: torch.Tensor, caches: Caches) -> torch.Tensor:
        """One new token for each document: rows x [docs][width]; the caches grow by one key."""
        if caches.longest >= caches.room:
            raise ValueError(f"caches of {caches.room} keys are full")
        docs = len(caches.length)
        at = (caches.start[:-1] + caches.length).long()
        caches.length += 1
        caches.longest += 1
        one = torch.arange(docs + 1, device=self.device, dtype=torch.int32)

        def attend(i, q, k, v):
            caches.k[i][at], caches.v[i][at] = k, v
            return B.attention(q, caches.k[i], caches.v[i], one, caches.start, 1, caches.longest, k_len=caches.length,
                               prefix=caches.prefix, causal=True, cap=self.config.cap)

        return self._run(x, attend)


def main() -> None:
    from . import net, scenes

    dev = torch.device("cuda:0")
    cloud = torch.from_numpy(scenes.workload(4).coords).to(dev)
    unet = net.Network(cloud, torch.bfloat16)
    x0 = torch.randn((len(cloud), net.STEM_C), device=dev).to(torch.bfloat16)
    level = 4
    tokens = unet.forward(x0, keep=True)[f"enc{level}"]
    coords = unet.coords[level]
    start, longest = documents(coords)
    model = Transformer(Config(width=tokens.shape[1]))
    seen = model.forward(tokens, start, longest, coords, spacing=1 << level)
    length = start[1:] - start[:-1]
    _, caches = model.prefill(seen, start, longest, longest + 16, prefix=length.contiguous())
    x = torch.randn((len(length), tokens.shape[1]), device=dev).to(torch.bfloat16)
    for _ in range(10):
        x = model.step(x, caches)
    torch.cuda.synchronize()
    print(f"{len(cloud)} voxels, {len(coords)} tokens in {len(length)} scenes, 10 new tokens each; "
          f"rms of the last {float(x.float().square().mean().sqrt()):.3f}")


if __name__ == "__main__":
    main()
