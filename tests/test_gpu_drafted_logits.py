"""What the decoder says of a token does not depend on how many are fed with it: the logits
of drafted steps, whose guesses are right in part, beside those of the same tokens fed one
by one.

Both compute in fp32 between the roundings of queries, keys and values to bf16 (and of keys
after they are turned; INT8: to its codes), which turn the other way where a sum of another
order lies beside a border: three roundings in each of two layers, 2^-8 of a value each, or for
INT8's codes and scales 2^-6, so 6 times that of a logit row's norm if all of them did.
A key at a wrong place, a guess that was not taken back, or a token that is seen too early
changes what attention adds, about as large as the rest.
"""
import pytest
import torch

from paper_2605_20600_amd import drafted
from paper_2605_20600_amd.best_of import Decoder, Shape

pytestmark = pytest.mark.gpu
IMAGES, STEPS, ROW = 3, 50, 7


def _sequences(vocab):
    """Images whose rows are copies of the row above but for a few tokens."""
    g = torch.Generator().manual_seed(5)
    new = torch.randint(1, vocab, (IMAGES, STEPS + 20), generator=g).tolist()
    for seq in new:
        for p in range(ROW, len(seq)):
            if p % 11 != 3:
                seq[p] = seq[p - ROW]
    return new


def _run(monkeypatch, decoder, prompt, drafts, kv, sequences):
    """Logits of each (image, token) when the images turn out to be `sequences`; most tokens
    gained in a step."""
    done, seen, most = [0] * IMAGES, {}, [0]

    def verify(logits, tokens, uniforms, counts=None, temperature=1.0):
        places = logits.shape[1]
        kept = torch.full((IMAGES, places), -1, dtype=torch.int32)
        count = torch.zeros(IMAGES, dtype=torch.int32)
        guess = tokens.tolist()
        left_out = [False] * IMAGES if counts is None else (counts < 0).tolist()
        for i, seq in enumerate(sequences):
            if left_out[i]:
                continue
            n = 0
            while n < places - 1 and guess[i][n] == seq[done[i] + n]:
                n += 1
            for j in range(n + 1):
                seen[i, done[i] + j] = logits[i, j].double().cpu()
                kept[i, j] = seq[done[i] + j]
            done[i] += n + 1
            count[i] = n + 1
            most[0] = max(most[0], n + 1)
        return {"tokens": kept.cuda(), "count": count.cuda(),
                "logprob": torch.zeros((IMAGES, places), device="cuda")}
    monkeypatch.setattr(drafted, "verify_drafts", verify)
    got = drafted.generate(decoder, prompt, IMAGES, STEPS, drafts, ROW, kv)
    assert got["tokens"].tolist() == [s[:STEPS] for s in sequences]
    return seen, most[0]


@pytest.mark.parametrize("kv,drafts,prompt", (("bf16", 4, 40), ("int8", 9, 5), ("bf16", 1, 300)))
def test_logits_of_drafted_steps(monkeypatch, kv, drafts, prompt):
    shape = Shape(vocab=300, layers=2, kv_heads=4, group=2, head_dim=64, local_heads=2, window=20,
                  page_tokens=32)
    decoder = Decoder(shape, seed=1)
    tokens = torch.randint(0, 300, (prompt,), generator=torch.Generator().manual_seed(2)).cuda()
    sequences = _sequences(300)
    alone, one = _run(monkeypatch, decoder, tokens, 0, kv, sequences)
    together, most = _run(monkeypatch, decoder, tokens, drafts, kv, sequences)
    assert one == 1 and most > min(drafts, 4)
    bound = 6 * 2.0 ** (-8 if kv == "bf16" else -6)
    for key in [(i, p) for i in range(IMAGES) for p in range(STEPS)]:
        a, b = alone[key], together[key]
        assert float((a - b).norm()) <= bound * float(a.norm()), key
