"""Images of one prompt decoded several tokens at a time: guesses copied from the row
above, verified against the decoder's own probabilities.

    python -m paper_2605_20600_amd.drafted --images 16 --steps 256 --drafts 4

Each step feeds the last token of every image and its guesses.  Queries and keys are
normalised and turned on their way into the cache, attention takes all of an image's
new tokens at once, and the verification says how many of them it keeps; lengths,
windows and page tables follow on the GPU, so that no step waits for the host.  What
comes out is distributed as if every token had been sampled alone.  The decoder has
random weights: there are no checkpoints here.
"""
from __future__ import annotations

import argparse
from typing import Dict

import torch

from .best_of import Decoder, Shape
from .drafts import verify_drafts
from .page_tables import PageTables
from .paged import PagedKV
from .rotary import Rotary

PIECE = 256  # prompt tokens that are attended at once


def generate(decoder: Decoder, prompt: torch.Tensor, images: int, steps: int, drafts: int = 4,
             row_len: int = 24, kv: str = "int8", temperature: float = 1.0, seed: int = 0
             ) -> Dict[str, torch.Tensor]:
    """`steps` tokens of `images` images after prompt (int64 [tokens], on the GPU), images
    being row_len tokens wide.  Returns "tokens" and "logprob" [images][steps], "passes", the
    times that the decoder has run, and "order": the images, the most probable first.
    RuntimeError where the decoder's logits give an image no next token (NaN, +inf, or all
    -inf)."""
    if prompt.dim() != 1 or len(prompt) < 1 or images < 1 or steps < 1 or drafts < 0 \
            or row_len < 1:
        raise ValueError("prompt must be [tokens], and tokens, images, steps and row_len at least "
                         f"1, drafts 0, got {tuple(prompt.shape)}, {images}, {steps}, {row_len} "
                         f"and {drafts}")
    with torch.cuda.device(prompt.device):
        return _generate(decoder, prompt, images, steps, drafts, row_len, kv, temperature, seed)


def _generate(decoder, prompt, images, steps, drafts, row_len, kv, temperature, seed):
    s, device, p = decoder.shape, prompt.device, decoder.shape.page_tokens
    places = drafts + 1
    prompt_pages, own_pages = -(-len(prompt) // p), -(-(steps + 2 * places) // p)
    window = torch.zeros((s.layers * images, s.kv_heads), dtype=torch.int32, device=device)
    window[:, :s.local_heads] = s.window
    # pages 0 .. are the images', the prompt's lie behind them
    own = s.layers * images * s.kv_heads * own_pages
    shared = s.layers * s.kv_heads * prompt_pages
    cache = PagedKV(kv, s.head_dim, s.kv_heads, own + shared, page_tokens=p, group=s.group,
                    device=device)
    tables = PageTables(s.kv_heads, own_pages, own, rows=images, layers=s.layers, page_tokens=p,
                        window=window, device=device)
    lists = [tables.lists(layer, max_len=steps + places) for layer in range(s.layers)]
    table = torch.arange(own, own + shared, dtype=torch.int32, device=device).view(
        s.layers, 1, s.kv_heads, prompt_pages)
    prompts = [cache.lists(table[layer], None, max_len=0) for layer in range(s.layers)]
    share = torch.zeros(images, dtype=torch.int32, device=device)
    rotary = Rotary(s.head_dim, norm="rms", device=str(device))

    def forward(tokens, positions, at, **kw):
        """Logits of tokens [rows][n] that join the lists `at`."""
        x = decoder.embed[tokens]
        rows, n = tokens.shape
        for layer in range(s.layers):
            q, k, v = decoder.project(layer, x.view(rows * n, -1))
            q, k, v = (t.view(rows, n, -1, s.head_dim) for t in (q, k, v))
            q = cache.write_rotary(at[layer], rotary, q, k, v, positions)
            o = cache.attn_tokens(at[layer], q, **(dict(kw, shared=prompts[layer]) if kw else {}),
                                  window=window[:rows] if kw else None)
            x = x + (o.view(rows * n, -1) @ decoder.out[layer]).view(x.shape)
        return x @ decoder.head

    place = torch.arange(len(prompt), dtype=torch.int32, device=device)[None]
    for begin in range(0, len(prompt), PIECE):
        piece = slice(begin, begin + PIECE)
        logits = forward(prompt[None, piece], place[:, piece].contiguous(), prompts)
        for l in prompts:
            l.advance(min(PIECE, len(prompt) - begin))

    g = torch.Generator(device=device).manual_seed(seed)
    width = steps + 2 * places
    tokens = torch.zeros((images, width), dtype=torch.int64, device=device)
    logprob = torch.zeros((images, width), device=device)
    done = torch.zeros(images, dtype=torch.int64, device=device)
    ahead = torch.arange(places, device=device)
    rows = torch.arange(images, device=device)[:, None]
    stuck = torch.zeros(images, dtype=torch.bool, device=device)  # no next token

    def keep(got):
        """Writes what was gained behind what is there; images that are done go nowhere."""
        stuck.logical_or_((got["count"] == 0) & (done < steps))
        at = (done[:, None] + ahead[:got["tokens"].shape[1]]).clamp(max=width - 1)
        tokens[rows, at] = got["tokens"].clamp(min=0).long()
        logprob[rows, at] = got["logprob"]
        done.add_(got["count"]).clamp_(max=steps + places)

    first = logits[:, -1:].expand(images, -1, -1)
    none = torch.zeros((images, 0), dtype=torch.int32, device=device)
    keep(verify_drafts(first, none, torch.rand((images, 1), generator=g, device=device),
                       temperature=temperature))
    passes, advance = 0, None
    while True:
        # (one look at the host every few steps, the first before any token is fed: a step
        # gains a token at least, but for images that have no next one)
        if passes % 8 == 0:
            least, *lost = torch.cat((done.min()[None], stuck)).tolist()
            if any(lost):
                raise RuntimeError("the decoder's logits give no next token for images "
                                   f"{[i for i, x in enumerate(lost) if x]}")
            if least >= steps:
                break
        tables.extend(places, advance=advance)
        above = done[:, None] - row_len + ahead[:drafts]  # the tokens over those to come
        guess = torch.where(above >= 0, tokens.gather(1, above.clamp(min=0)), 0)
        last = tokens.gather(1, done[:, None] - 1)
        fed = torch.cat((last, guess), 1)
        at = (len(prompt) + done[:, None] - 1 + ahead).to(torch.int32)
        logits = forward(fed, at, lists, share=share)
        got = verify_drafts(logits, guess.to(torch.int32),
                            torch.rand((images, places), generator=g, device=device),
                            counts=torch.where((done >= steps) | stuck, -1, drafts).to(torch.int32),
                            temperature=temperature)
        keep(got)
        advance = got["count"]
        passes += 1
    res = {"tokens": tokens[:, :steps], "logprob": logprob[:, :steps],
           "passes": torch.tensor(passes)}
    res["order"] = res["logprob"].sum(1).argsort(descending=True)
    return res


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--images", type=int, default=16)
    p.add_argument("--steps", type=int, default=256)
    p.add_argument("--drafts", type=int, default=4, help="tokens that are guessed at a time")
    p.add_argument("--row", type=int, default=24, help="tokens of an image's row")
    p.add_argument("--prompt", type=int, default=64, help="tokens of the (random) prompt")
    p.add_argument("--kv", choices=("bf16", "int8", "fp4"), default="int8")
    p.add_argument("--temperature", type=float, default=1.0)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args()
    shape = Shape()
    prompt = torch.randint(0, shape.vocab, (a.prompt,),
                           generator=torch.Generator().manual_seed(a.seed)).cuda()
    got = generate(Decoder(shape, a.seed), prompt, a.images, a.steps, a.drafts, a.row, a.kv,
                   a.temperature, a.seed)
    print(f"{a.steps} tokens of {a.images} images in {int(got['passes'])} passes")
    for place, image in enumerate(got["order"].tolist()):
        print(f"{place + 1}. image {image}: {float(got['logprob'][image].mean()):.4f} nats per token")


if __name__ == "__main__":
    main()
