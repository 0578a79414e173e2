"""Drafted images whose decoder gives no next token: an error within a few steps, before
anything is taken from a place that there is not."""
import math

import pytest
import torch

from paper_2605_20600_amd import drafted
from paper_2605_20600_amd.best_of import Decoder, Shape

pytestmark = pytest.mark.gpu
SHAPE = Shape(vocab=300, layers=2, kv_heads=4, group=2, head_dim=64, local_heads=2, window=20,
              page_tokens=32)


def _generate(decoder, **kw):
    tokens = torch.randint(0, 300, (5,), generator=torch.Generator().manual_seed(2)).cuda()
    return drafted.generate(decoder, tokens, **{**dict(images=3, steps=50, drafts=4, row_len=7,
                                                       seed=3), **kw})


@pytest.mark.parametrize("call", (0, 1, 7, 8, 13))
def test_an_image_without_a_next_token(monkeypatch, call):
    # verification number `call` (0: of the prompt's last token) ends image 1
    verify, calls, counts = drafted.verify_drafts, [], []

    def ends(*args, **kw):
        got = verify(*args, **kw)
        if len(calls) == call:
            got["tokens"][1], got["count"][1], got["logprob"][1] = -1, 0, 0
        calls.append(0)
        counts.append(kw.get("counts"))
        return got
    monkeypatch.setattr(drafted, "verify_drafts", ends)
    with pytest.raises(RuntimeError, match=r"images \[1\]"):
        _generate(Decoder(SHAPE, seed=1))
    # at the next look, of which there is one every eight steps; left out until then
    assert len(calls) == 1 + (call + 7) // 8 * 8
    assert all(int(c[1]) == -1 and int(c[0]) == 4 for c in counts[call + 1:])


@pytest.mark.parametrize("value", (math.nan, math.inf))
@pytest.mark.parametrize("temperature", (0.0, 1.0))
def test_logits_that_are_no_numbers(value, temperature):
    decoder = Decoder(SHAPE, seed=1)
    decoder.head[:, 7] = value
    with pytest.raises(RuntimeError, match=r"images \[0, 1, 2\]"):
        _generate(decoder, temperature=temperature)


def test_images_that_end_with_the_last_token():
    # one step and no drafts: nothing is fed after the prompt
    got = _generate(Decoder(SHAPE, seed=1), steps=1, drafts=0)
    assert got["tokens"].shape == (3, 1) and int(got["passes"]) == 0
