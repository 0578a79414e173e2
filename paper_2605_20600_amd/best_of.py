"""Several images of one prompt, ranked by the probability of their tokens: the
paged cache, its attention with a shared prefix and the token scores, as a
decoder uses them together.

    python -m paper_2605_20600_amd.best_of --images 16 --steps 256 --kv int8

The prompt's keys and values are written once, to lists that every image shares.
Each image has lists of its own; its local heads see a window of its last tokens,
and a page that falls behind the window is used again for what comes.  The decoder
has random weights: there are no checkpoints here.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass
from typing import Dict, List, Optional

import torch

from .paged import Lists, PagedKV, token_logprobs


@dataclass(frozen=True)
class Shape:
    vocab: int = 16384
    layers: int = 4
    kv_heads: int = 8
    group: int = 2      # query heads per kv head
    head_dim: int = 64
    local_heads: int = 4  # of the kv heads, the first ones
    window: int = 128     # tokens that a local head sees
    page_tokens: int = 64

    @property
    def width(self) -> int:
        return self.kv_heads * self.group * self.head_dim


class Decoder:
    """Attention layers with a residual between an embedding and its transpose."""

    def __init__(self, shape: Shape, seed: int = 0, device: str = "cuda"):
        g = torch.Generator().manual_seed(seed)
        w, kv = shape.width, shape.kv_heads * shape.head_dim
        self.shape = shape

        def normal(*dims, scale):
            return (torch.randn(dims, generator=g) * scale).to(device)

        self.embed = normal(shape.vocab, w, scale=1.0)
        self.qkv = [normal(w, w + 2 * kv, scale=w ** -0.5) for _ in range(shape.layers)]
        self.out = [normal(w, w, scale=w ** -0.5) for _ in range(shape.layers)]
        self.head = normal(w, shape.vocab, scale=2 * w ** -0.5)

    def project(self, layer: int, x: torch.Tensor):
        """q [rows][heads][d], k and v [rows][1][kv_heads][d], bf16."""
        s = self.shape
        kv = s.kv_heads * s.head_dim
        q, k, v = (x @ self.qkv[layer]).to(torch.bfloat16).split((s.width, kv, kv), dim=1)
        return (q.reshape(-1, s.kv_heads * s.group, s.head_dim),
                *(t.reshape(-1, 1, s.kv_heads, s.head_dim) for t in (k, v)))


class _Layer:
    """Lists of one layer: the prompt's and the images'."""

    def __init__(self, cache: PagedKV, shape: Shape, prompt: int, images: int, steps: int,
                 first_page: int):
        p = shape.page_tokens
        heads, local = shape.kv_heads, shape.local_heads
        prompt_pages, own_pages = -(-prompt // p), -(-steps // p)
        # a local head holds the pages that its window can touch, and takes them in turn
        self.held = min(own_pages, -(-shape.window // p) + 1)
        self.next_page = first_page

        def take(*dims):
            n = 1
            for x in dims:
                n *= x
            at = self.next_page
            self.next_page += n
            return torch.arange(at, at + n, dtype=torch.int32).view(*dims).to(cache.device)

        self.prompt = cache.lists(take(1, heads, prompt_pages), None, max_len=0)
        table = torch.full((images, heads, own_pages), -1, dtype=torch.int32, device=cache.device)
        table[:, local:] = take(images, heads - local, own_pages)
        table[:, :local, :self.held] = take(images, local, self.held)
        self.first = torch.zeros((images, heads), dtype=torch.int32, device=cache.device)
        self.own = cache.lists(table, None, max_len=0, first=self.first)

    def slide(self, shape: Shape) -> None:
        """Before the next token is written: the windows as they are with it."""
        p, length = shape.page_tokens, self.own.extra + 1
        if length > shape.window:
            self.first[:, :shape.local_heads] = length - shape.window
        page = (length - 1) // p
        if (length - 1) % p == 0 and page >= self.held:
            pages = self.own.pages[:, :shape.local_heads]
            pages[:, :, page] = pages[:, :, page - self.held]
            pages[:, :, page - self.held] = -1


def _pages(shape: Shape, prompt: int, images: int, steps: int) -> int:
    p = shape.page_tokens
    own = -(-steps // p)
    local = min(own, -(-shape.window // p) + 1)
    return shape.layers * (shape.kv_heads * -(-prompt // p) + images * (
        shape.local_heads * local + (shape.kv_heads - shape.local_heads) * own))


def generate(decoder: Decoder, prompt: torch.Tensor, images: int, steps: int, kv: str = "int8",
             temperature: float = 1.0, top: int = 0, seed: int = 0) -> Dict[str, torch.Tensor]:
    """`steps` tokens of `images` images after prompt (int64 [tokens], on the GPU).
    Returns "tokens" [steps][images] with their "logprob" and "entropy", with top > 0
    the alternatives' "top_logprob" and "top_index" [steps][images][top], and
    "order": the images, the most probable first."""
    if prompt.dim() != 1 or len(prompt) < 1 or images < 1 or steps < 1:
        raise ValueError("prompt must be [tokens], and tokens, images and steps at least 1, got "
                         f"{tuple(prompt.shape)}, {images} and {steps}")
    with torch.cuda.device(prompt.device):
        return _generate(decoder, prompt, images, steps, kv, temperature, top, seed)


def _generate(decoder: Decoder, prompt: torch.Tensor, images: int, steps: int, kv: str,
              temperature: float, top: int, seed: int) -> Dict[str, torch.Tensor]:
    s = decoder.shape
    device = prompt.device
    cache = PagedKV(kv, s.head_dim, s.kv_heads, _pages(s, len(prompt), images, steps),
                    page_tokens=s.page_tokens, group=s.group, device=device)
    layers: List[_Layer] = []
    for _ in range(s.layers):
        layers.append(_Layer(cache, s, len(prompt), images, steps,
                             layers[-1].next_page if layers else 0))
    share = torch.zeros(images, dtype=torch.int32, device=device)

    def forward(x: torch.Tensor, lists: List[Lists], shared: Optional[List[Lists]]) -> torch.Tensor:
        for i, l in enumerate(lists):
            q, k, v = decoder.project(i, x)
            cache.write(l, k, v)
            l.advance()
            o = cache.attn(l, q) if shared is None else cache.attn(l, q, shared=shared[i],
                                                                   share=share)
            x = x + o.view(len(x), -1) @ decoder.out[i]
        return x

    # the prompt is attended token by token, as an image of its own
    for token in prompt:
        x = forward(decoder.embed[token][None], [l.prompt for l in layers], None)
    x = x.expand(images, -1)

    g = torch.Generator(device=device).manual_seed(seed)
    found: Dict[str, List[torch.Tensor]] = {}
    for step in range(steps):
        logits = x @ decoder.head
        noise = torch.rand(logits.shape, generator=g, device=device)
        tokens = (logits / temperature - (-noise.clamp_min(1e-20).log()).log()).argmax(1)
        got = token_logprobs(logits, tokens.to(torch.int32), top=top, temperature=temperature)
        for name, t in dict(got, tokens=tokens).items():
            found.setdefault(name, []).append(t)
        if step + 1 < steps:
            for l in layers:
                l.slide(s)
            x = forward(decoder.embed[tokens], [l.own for l in layers], [l.prompt for l in layers])
    res = {name: torch.stack(t) for name, t in found.items()}
    res["order"] = res["logprob"].sum(0).argsort(descending=True)
    return res


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--images", type=int, default=16)
    p.add_argument("--steps", type=int, default=256)
    p.add_argument("--prompt", type=int, default=64, help="tokens of the (random) prompt")
    p.add_argument("--kv", choices=("bf16", "int8", "fp4"), default="int8")
    p.add_argument("--temperature", type=float, default=1.0)
    p.add_argument("--top", type=int, default=5, help="alternatives of each token")
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args()
    shape = Shape()
    prompt = torch.randint(0, shape.vocab, (a.prompt,),
                           generator=torch.Generator().manual_seed(a.seed)).cuda()
    got = generate(Decoder(shape, a.seed), prompt, a.images, a.steps, a.kv, a.temperature, a.top,
                   a.seed)
    logprob, entropy = got["logprob"].mean(0), got["entropy"].mean(0)
    for place, image in enumerate(got["order"].tolist()):
        print(f"{place + 1}. image {image}: {float(logprob[image]):.4f} nats per token, "
              f"entropy {float(entropy[image]):.4f}, mean rank "
              f"{float(got['rank'][:, image].float().mean()):.1f}")


if __name__ == "__main__":
    main()
