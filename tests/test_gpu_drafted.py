"""The operators of a drafted step together: what a list holds after many steps, whose
guesses were kept in part, is bit for bit what it would hold had the kept tokens been
written alone; attention over it, page by page, is that over a list of its own; the command
runs."""
import pytest
import torch

from paper_2605_20600_amd import drafted
from paper_2605_20600_amd.best_of import Decoder, Shape
from paper_2605_20600_amd.drafts import verify_drafts
from paper_2605_20600_amd.page_tables import PageTables
from paper_2605_20600_amd.paged import PagedKV
from paper_2605_20600_amd.rotary import NormWeights, Rotary

pytestmark = pytest.mark.gpu


class Model:
    """Queries, keys and values that follow from a token and its place alone, so that what was
    fed beside a token leaves no trace; logits that follow from the token before."""

    def __init__(self, vocab, heads, group, d, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.qkv = torch.randn((vocab, (group + 2) * heads, d), generator=g,
                               device="cuda").bfloat16()
        self.next = 2.0 * torch.randn((vocab, vocab), generator=g, device="cuda")
        self.heads, self.group = heads, group

    def __call__(self, tokens):
        x = self.qkv[tokens]
        return x.split((self.group * self.heads, self.heads, self.heads), dim=2)


@pytest.mark.parametrize("kv", ("bf16", "int8", "fp4"))
@pytest.mark.parametrize("drafts,rows", ((0, 3), (4, 6), (9, 40)))
def test_steps_together(kv, drafts, rows):
    vocab, heads, group, d, steps, ptok = 24, 4, 2, 64, 14, 32
    places, layers = drafts + 1, 2
    model = Model(vocab, heads, group, d)
    window = torch.tensor([0, 40, 0, 7], dtype=torch.int32, device="cuda").repeat(rows * layers, 1)
    most = -(-(steps + 2) * places // ptok)
    pages = rows * layers * heads * most
    cache = PagedKV(kv, d, heads, pages, page_tokens=ptok, group=group)
    cache.pool.fill_(255)
    tables = PageTables(heads, most, pages, rows, layers, page_tokens=ptok, window=window)
    lists = [tables.lists(layer) for layer in range(layers)]
    rotary = Rotary(d, 32, layout="pairs", norm="rms")
    w = NormWeights(torch.rand(d, device="cuda") + 0.5, None, torch.rand((heads, d), device="cuda"))
    g = torch.Generator(device="cuda").manual_seed(1)
    kept = torch.zeros((rows, steps * places + 2), dtype=torch.int64, device="cuda")
    done = torch.ones(rows, dtype=torch.int64, device="cuda")  # the first token is 0
    advance, at = None, torch.arange(places, device="cuda")
    total = 0
    for step in range(steps):
        tables.extend(places, advance=advance)
        last = kept.gather(1, done[:, None] - 1)
        guess = torch.randint(0, vocab, (rows, drafts), generator=g, device="cuda")
        if drafts:  # good guesses too
            best = model.next[last[:, 0]].argmax(1)
            guess[:, 0] = torch.where(torch.arange(rows, device="cuda") % 2 == 0, best, guess[:, 0])
        fed = torch.cat((last, guess), 1)
        position = (done[:, None] - 1 + at).to(torch.int32)
        q, k, v = model(fed)
        for layer in range(layers):
            turned = cache.write_rotary(lists[layer], rotary, q, k, v, position, weights=w)
            out = cache.attn_tokens(lists[layer], turned, window=window[:rows])
        got = verify_drafts(model.next[fed], guess.to(torch.int32),
                            torch.rand((rows, places), generator=g, device="cuda"))
        assert bool((got["count"] >= 1).all()) and bool((got["count"] <= places).all())
        there = at < got["count"][:, None]
        assert bool(((got["tokens"] >= 0) == there).all())
        kept.scatter_(1, done[:, None] + at, got["tokens"].clamp(min=0).long())
        # each kept one is a guess, but for the last
        same = got["tokens"][:, :drafts] == guess
        assert bool((same | (at[:drafts] >= got["count"][:, None] - 1)).all())
        done += got["count"]
        advance = got["count"]
        total += int(got["count"].sum())
        assert int(tables.free_state[2]) == 0
    assert drafts == 0 or total > rows * steps  # some were kept
    tables.extend(0, advance=advance)
    length = done - 1  # fed tokens whose keys and values count
    assert torch.equal(tables.len, length.to(torch.int32).repeat(layers)[:, None].expand(-1, heads))
    # the same tokens alone, in lists of their own
    n = int(length.max())
    fresh = PagedKV(kv, d, heads, rows * heads * most, page_tokens=ptok, group=group)
    alone = torch.randperm(rows * heads * most).to(torch.int32).view(rows, heads, most).cuda()
    q, k, v = model(kept[:, :n])
    position = torch.arange(n, dtype=torch.int32, device="cuda").repeat(rows, 1)
    turned, key = rotary(q, k, position, weights=w)
    empty = fresh.lists(alone, None, max_len=0)
    fresh.write(empty, key, v.contiguous(), counts=length.to(torch.int32))
    same = fresh.lists(alone, tables.len[:rows].contiguous(), max_len=most * ptok)
    want = fresh.read(same, n)
    for layer in range(layers):
        got = cache.read(lists[layer], n)
        seen = torch.arange(n, device="cuda")[None, :, None] >= tables.first[:rows][:, None]
        for a, b in zip(got, want):
            assert torch.equal(torch.where(seen[..., None], a, 0), torch.where(seen[..., None], b, 0))
    # and what the last kept tokens attend: the same bits again (same lists, same launch)
    one = turned.gather(1, (length - 1)[:, None, None, None].expand(-1, 1, heads * group, d))
    back = torch.ones((), dtype=torch.int32, device="cuda")
    before = [(tables.pages[:rows], cache), (alone, fresh)]
    outs = [c.attn_tokens(c.lists(p.contiguous(), (tables.len[:rows] - back).contiguous(),
                                  max_len=most * ptok), one, window=window[:rows])
            for p, c in before]
    # (pages behind a window are gone from the first)
    assert torch.equal(*outs)


@pytest.mark.parametrize("kv,drafts,prompt", (("int8", 4, 5), ("fp4", 0, 1), ("bf16", 7, 300)))
def test_the_command(kv, drafts, prompt):
    shape = Shape(vocab=300, layers=2, kv_heads=4, group=2, head_dim=64, local_heads=2, window=20,
                  page_tokens=32)
    decoder = Decoder(shape, seed=1)
    tokens = torch.randint(0, 300, (prompt,), generator=torch.Generator().manual_seed(2)).cuda()
    got = drafted.generate(decoder, tokens, images=3, steps=50, drafts=drafts, row_len=7, kv=kv,
                           temperature=0.7, seed=3)
    assert got["tokens"].shape == (3, 50) and got["logprob"].shape == (3, 50)
    assert bool(((got["tokens"] >= 0) & (got["tokens"] < 300)).all())
    assert bool((got["logprob"] < 0).all()) and bool(got["logprob"].isfinite().all())
    assert sorted(got["order"].tolist()) == [0, 1, 2]
    again = drafted.generate(decoder, tokens, images=3, steps=50, drafts=drafts, row_len=7, kv=kv,
                             temperature=0.7, seed=3)
    assert torch.equal(got["tokens"], again["tokens"])
    for bad in (dict(images=0), dict(steps=0), dict(drafts=-1), dict(row_len=0)):
        with pytest.raises(ValueError):
            drafted.generate(decoder, tokens, **{**dict(images=1, steps=1), **bad})
