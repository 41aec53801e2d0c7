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
one new token for each document a call.  ``extend`` is for documents that come and go and grow by any
number of tokens a call, prompts in chunks and single tokens together: their caches are pages, in the
rows' type or in 8 bits.

Between the first product and attention, where the configuration asks for it:

  q, k = norm of each head, turned by their places or voxels    spconv_rotate_heads
  pages <- k, v                                                 spconv_cache_write
  o     = attention(q, pages)                                   spconv_cached_attention

    python -m paper_2401_06145_amd.transformer      # a small UNet encoder, its voxels, ten new tokens
"""
from __future__ import annotations

from dataclasses import dataclass, field

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
    head_norm: bool = False   # norms of queries and keys for each head
    rotary: int = 0           # columns of a head that turn by place, or by the voxel's coordinates; 0: none
    base: float = 10_000.0    # of the frequencies
    factor: float = 1.0       # for contexts that many times longer than ``trained`` (binding.rotary_frequencies)
    trained: int = 0

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


@dataclass
class PagedCaches:
    """Keys and values of each layer in pages that all documents share out among them; the same table for
    every layer.  Lengths are known to the host, which gives pages out as documents grow."""
    layers: list              # of B.Pages
    table: torch.Tensor       # int32 [docs][most pages of one]
    length: torch.Tensor      # int32 [docs]
    lens: list                # the same, on the host
    free: list                # pages of no document
    dtype: torch.dtype
    prefix: torch.Tensor | None = None
    held: list = field(default_factory=list)  # pages of each document, in order

    @property
    def page(self) -> int:
        return self.layers[0].page

    def grow(self, new: list) -> None:
        """Room for new[t] more tokens of each document t; all of it or, where pages run out, none."""
        if len(new) != len(self.lens) or any(n < 0 for n in new):
            raise ValueError(f"expected {len(self.lens)} numbers of new tokens, got {new}")
        lens = [a + b for a, b in zip(self.lens, new)]
        more = [-(-n // self.page) - len(p) for n, p in zip(lens, self.held)]
        if max(lens, default=0) > self.table.shape[1] * self.page:
            raise ValueError(f"a document of {max(lens)} tokens does not fit {self.table.shape[1]} pages of {self.page}")
        if sum(more) > len(self.free):
            raise ValueError(f"{sum(more)} more pages are needed, and {len(self.free)} are free")
        at = []
        for t, m in enumerate(more):
            at.extend(t * self.table.shape[1] + len(self.held[t]) + i for i in range(m))
        of = self.free[:-len(at) - 1:-1]  # from the end, as they are given out
        if at:
            both = torch.tensor([at, of], dtype=torch.int64).to(self.table.device)
            self.table.view(-1)[both[0]] = both[1].to(torch.int32)
        self.length += torch.tensor(new, dtype=torch.int32).to(self.length.device)
        # the host's side last: what raised above has changed nothing that a call reads
        del self.free[len(self.free) - len(at):]
        for t, m in enumerate(more):
            self.held[t].extend(of[:m])
            del of[:m]
        self.lens = lens

    def shrink(self, new: list) -> None:
        """Takes the last new[t] tokens of each document t back, as if they had not come."""
        self.length -= torch.tensor(new, dtype=torch.int32).to(self.length.device)
        self.lens = [a - b for a, b in zip(self.lens, new)]
        for held, n in reversed(list(zip(self.held, self.lens))):
            while len(held) > -(-n // self.page):
                self.free.append(held.pop())

    def release(self, doc: int) -> None:
        """Document ``doc`` ends: its pages are free, and its place is an empty document's."""
        self.free.extend(reversed(self.held[doc]))
        self.held[doc], self.lens[doc] = [], 0
        self.length[doc] = 0
        if self.prefix is not None:
            self.prefix[doc] = 0

    def read(self, layer: int) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """(keys, values, first row of each document) of one layer, packed as ``attention`` takes them."""
        start = torch.tensor([sum(self.lens[:t]) for t in range(len(self.lens) + 1)], dtype=torch.int32).to(self.table.device)
        k, v = B.cache_read(self.layers[layer], start, self.table, sum(self.lens), self.dtype)
        return k, v, start


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
        if c.head_norm:
            for w in self.layers:
                w["g_q"], w["g_k"] = gamma(c.head_dim), gamma(c.head_dim)
        self.freq, self.gain = B.rotary_frequencies(c.rotary, c.base, c.factor, c.trained, device=self.device)
        self.slopes = torch.exp2(-8.0 * torch.arange(1, c.heads + 1) / c.heads).to(self.device)

    def _linear(self, rows, weight, relu=False):
        return B.scaled_linear(rows[0], rows[1], weight[0], weight[1], self.dtype, relu=relu, exact=self.config.exact)

    def _places(self, n: int, start: torch.Tensor, first: torch.Tensor | None = None) -> torch.Tensor | None:
        """Each of n rows' place in its document, whose rows begin at place ``first`` (0)."""
        if not (self.config.rotary or self.config.head_norm):
            return None
        row = torch.arange(n, device=self.device)
        doc = torch.searchsorted(start[1:].contiguous(), row, right=True).clamp(max=len(start) - 2)
        place = row - start[doc]
        return (place if first is None else place + first[doc]).to(torch.int32)

    def _run(self, x: torch.Tensor, attend, pos: torch.Tensor | None = None) -> torch.Tensor:
        """The layers on rows x; attend(layer, q, k, v) is their attention; pos: the rows' places or voxels."""
        c = self.config
        kv = c.kv_heads * c.head_dim
        add = None
        for i, w in enumerate(self.layers):
            *a, total = B.rms_norm(x, w["g_in"], residual=add, eps=c.eps, bits8=True)
            x = x if add is None else total
            q, k, v = (t.unflatten(1, (-1, c.head_dim)) for t in self._linear(a, w["qkv"]).split([c.width, kv, kv], 1))
            if c.rotary or c.head_norm:
                q, k = B.rotate_heads(q, k, pos, self.freq, w.get("g_q"), w.get("g_k"), eps=c.eps, gain=self.gain)
            o = attend(i, q, k, v).flatten(1)
            add = self._linear(B.rms_norm(o, w["g_out"], eps=c.eps, bits8=True)[:2], w["out"])
            *a, x = B.rms_norm(x, w["g_up"], residual=add, eps=c.eps, bits8=True)
            u = self._linear(a, w["up"], relu=True)
            add = self._linear(B.rms_norm(u, w["g_down"], eps=c.eps, bits8=True)[:2], w["down"])
        return B.rms_norm(x, self.g_last, residual=add, eps=c.eps)[0]

    def forward(self, x: torch.Tensor, start: torch.Tensor, longest: int, coords: torch.Tensor | None = None,
                causal: bool = False, prefix: torch.Tensor | None = None, spacing: int = 1) -> torch.Tensor:
        """Whole documents: rows x [n][width], document t being rows start[t] .. start[t + 1].  With
        coords, scores fall with the voxels' distance, in units of ``spacing`` (the level's), and heads
        turn, if they do, by the voxels' coordinates."""
        slopes = None if coords is None else self.slopes / spacing
        return self._run(x, lambda i, q, k, v: B.attention(
            q, k, v, start, start, longest, longest, prefix=prefix, causal=causal, cap=self.config.cap, slopes=slopes,
            q_pos=coords, k_pos=coords), self._places(len(x), start) if coords is None else coords)

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

        return self._run(x, attend, self._places(len(x), start)), caches

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

        return self._run(x, attend, (caches.length - 1).contiguous())

    def pages(self, docs: int, pages: int, page: int = 64, bits8: bool = False, most: int | None = None,
              prefix: torch.Tensor | None = None) -> PagedCaches:
        """Caches of ``pages`` pages a layer for ``docs`` documents, empty ones, of up to ``most`` pages each."""
        c = self.config
        return PagedCaches([B.Pages.make(pages, page, c.kv_heads, c.head_dim, self.dtype, bits8, self.device) for _ in range(c.layers)],
                           torch.full((docs, most or pages), -1, dtype=torch.int32, device=self.device),
                           torch.zeros(docs, dtype=torch.int32, device=self.device), [0] * docs, list(range(pages))[::-1],
                           self.dtype, None if prefix is None else prefix.clone(), [[] for _ in range(docs)])

    def extend(self, x: torch.Tensor, new: list, caches: PagedCaches) -> torch.Tensor:
        """New tokens for each document, any number (a prompt, its next chunk, one token, none): rows
        x [sum(new)][width] in the documents' order; the caches grow by them, or, where the call raises, stay as
        they were.  Tokens see of their document's prefix what has come with this call: a prefix that all of
        it should see comes in one.  Heads turn by place (voxels are ``forward``'s)."""
        if len(x) != sum(new):
            raise ValueError(f"{sum(new)} new tokens, but {len(x)} rows")
        if len(x) and (x.dim() != 2 or x.shape[1] != self.config.width or x.dtype != self.dtype or x.device != caches.table.device):
            raise ValueError(f"x: expected {self.dtype} rows of {self.config.width} on {caches.table.device}, got {x.dtype} "
                             f"{tuple(x.shape)} on {x.device}")
        first = caches.length.clone()
        caches.grow(new)
        try:
            return self._extend(x, new, caches, first) if len(x) else x
        except BaseException:
            caches.shrink(new)
            raise

    def _extend(self, x: torch.Tensor, new: list, caches: PagedCaches, first: torch.Tensor) -> torch.Tensor:
        start = torch.tensor([sum(new[:t]) for t in range(len(new) + 1)], dtype=torch.int32).to(self.device)

        def attend(i, q, k, v):
            B.cache_write(caches.layers[i], k, v, start, caches.length, caches.table)
            return B.cached_attention(q, caches.layers[i], start, caches.length, caches.table, max(new), max(caches.lens),
                                      prefix=caches.prefix, cap=self.config.cap)

        return self._run(x, attend, self._places(len(x), start, first))


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
    # the same scenes, turned by place, as documents in 8-bit pages: a chunk of voxels at a time, then new tokens
    turned = Transformer(Config(width=tokens.shape[1], head_norm=True, rotary=tokens.shape[1] // 8))
    lens = length.tolist()
    paged = turned.pages(len(lens), sum(-(-(n + 10) // 64) for n in lens), bits8=True)
    for at in range(0, longest, 1024):
        chunk = [max(0, min(1024, n - at)) for n in lens]
        rows = torch.cat([tokens[int(start[t]) + at:int(start[t]) + at + n] for t, n in enumerate(chunk)])
        y = turned.extend(rows, chunk, paged)
    y = torch.randn((len(lens), tokens.shape[1]), device=dev).to(torch.bfloat16)
    for _ in range(10):
        y = turned.extend(y, [1] * len(lens), paged)
    keys, _, _ = paged.read(0)
    torch.cuda.synchronize()
    print(f"in pages: {len(keys)} keys a layer, rms {float(keys.float().square().mean().sqrt()):.3f}; "
          f"rms of the last tokens {float(y.float().square().mean().sqrt()):.3f}")
    print(f"{len(cloud)} voxels, {len(coords)} tokens in {len(length)} scenes, 10 new tokens each; "
          f"rms of the last {float(x.float().square().mean().sqrt()):.3f}")


if __name__ == "__main__":
    main()
