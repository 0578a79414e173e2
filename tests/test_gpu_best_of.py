"""Several images of one prompt, against a plain 64-bit decoder with the same
tokens: dense keys and values in place of pages, windows by a mask.

Both round queries, keys and values to bf16; where the two disagree on one it is by
an ulp, 2^-8 of the number at most.  If all of them did, the weighted means would be
off by 2^-8 from the values and by 2^-7 |score| from the scores, relatively, and so
would each layer's part of the sum that the logits are products of.  The scores here
are q . k / sqrt(d) with components of order one: under 8.  So a logit is off by at
most layers * (2^-8 + 8 * 2^-7) * its sum's largest term, in the mean over the width
far less; a tenth of that bound is asked for, on log probabilities of order ten.
"""
import math

import pytest
import torch

from paper_2605_20600_amd.best_of import Decoder, Shape, generate

pytestmark = pytest.mark.gpu


def _bf16(x):
    return x.to(torch.bfloat16).double()


def _plain(decoder, prompt, tokens, temperature):
    """Log probability and entropy [steps][images] of given tokens."""
    s = decoder.shape
    kv = s.kv_heads * s.head_dim
    embed, head = decoder.embed.double().cpu(), decoder.head.double().cpu()
    qkv, out = ([w.double().cpu() for w in ws] for ws in (decoder.qkv, decoder.out))
    logprob = torch.zeros(tokens.shape, dtype=torch.float64)
    entropy = torch.zeros_like(logprob)
    for image in range(tokens.shape[1]):
        cache = [([], []) for _ in range(s.layers)]
        n = 0

        def forward(token):
            x = embed[token]
            for i in range(s.layers):
                y = _bf16((x @ qkv[i]).float())
                q = y[:s.width].view(s.kv_heads, s.group, s.head_dim)
                cache[i][0].append(y[s.width:s.width + kv].view(s.kv_heads, s.head_dim))
                cache[i][1].append(y[s.width + kv:].view(s.kv_heads, s.head_dim))
                k, v = (torch.stack(c, 1) for c in cache[i])  # [heads][tokens][d]
                sc = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(s.head_dim)
                at = torch.arange(k.shape[1]) - len(prompt)
                gone = (at >= 0) & (at < n - s.window)  # n: the image's tokens so far
                sc[:s.local_heads, :, gone] = -math.inf
                x = x + torch.matmul(sc.softmax(-1), v).reshape(-1) @ out[i]
            return x

        for t in prompt.tolist():
            x = forward(t)
        for step in range(tokens.shape[0]):
            lp = (x @ head / temperature).log_softmax(0)
            logprob[step, image] = lp[tokens[step, image]]
            entropy[step, image] = -(lp.exp() * lp).sum()
            n = step + 1
            if n < tokens.shape[0]:
                x = forward(tokens[step, image])
    return logprob, entropy


def test_images_of_a_prompt():
    shape = Shape(vocab=500, layers=2, kv_heads=4, group=2, head_dim=64, local_heads=2, window=40,
                  page_tokens=32)
    decoder = Decoder(shape, seed=1)
    prompt = torch.randint(0, shape.vocab, (37,), generator=torch.Generator().manual_seed(2)).cuda()
    got = generate(decoder, prompt, images=3, steps=150, kv="bf16", temperature=0.8, top=4, seed=3)
    want, want_entropy = _plain(decoder, prompt, got["tokens"].cpu(), 0.8)
    tol = 0.1 * shape.layers * (2.0 ** -8 + 8 * 2.0 ** -7) * 10
    assert float((got["logprob"].cpu() - want).abs().max()) <= tol
    assert float((got["entropy"].cpu() - want_entropy).abs().max()) <= tol
    assert got["top_logprob"].shape == (150, 3, 4)
    assert bool((got["top_logprob"][..., 0] >= got["logprob"]).all())
    total = got["logprob"].sum(0)[got["order"]]
    assert bool((total[:-1] >= total[1:]).all())


@pytest.mark.parametrize("kv", ("int8", "fp4"))
def test_every_cache_type(kv):
    shape = Shape(vocab=1000, layers=2, window=64)
    got = generate(Decoder(shape, seed=4), torch.arange(70, device="cuda"), images=5, steps=140,
                   kv=kv)
    assert got["tokens"].shape == (140, 5) and bool(got["logprob"].isfinite().all())
    assert sorted(got["order"].tolist()) == list(range(5))
