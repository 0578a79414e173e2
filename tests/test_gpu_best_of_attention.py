"""Every attention call that best_of makes, for each type of cache, against 64 bits over
the queries, keys and values that it was given: pages taken in turn by windows, lists
that grow, the prompt that images share.  Bounds as in test_gpu_paged.py."""
import pytest
import torch

from paper_2605_20600_amd import best_of
from paper_2605_20600_amd.best_of import Decoder, Shape, generate
from paper_2605_20600_amd.paged import PagedKV
from test_gpu_paged import TYPES, U, _held, _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("window,page", ((64, 64), (40, 32), (100, 32)))
def test_attention_of_a_generation(kind, window, page, monkeypatch):
    shape = Shape(vocab=300, layers=2, kv_heads=4, group=2, head_dim=64, local_heads=2,
                  window=window, page_tokens=page)
    written, calls = {}, []  # keys and values by lists; (own, shared, tokens of own, q, out)

    class Recorded(PagedKV):
        def write(self, lists, k, v, counts=None):
            written.setdefault(id(lists), []).append((k.cpu(), v.cpu()))
            super().write(lists, k, v, counts)

        def attn(self, own, q, **kw):
            lse = torch.empty(q.shape[:2], device=q.device)
            out = super().attn(own, q, lse=lse, **kw)
            shared = kw.get("shared")
            calls.append((id(own), None if shared is None else id(shared), len(written[id(own)]),
                          q.cpu(), out.cpu().double(), lse.cpu().double()))
            return out

    monkeypatch.setattr(best_of, "PagedKV", Recorded)
    images, steps, prompt = 3, 210, 37
    generate(Decoder(shape, seed=1), torch.arange(prompt, device="cuda"), images, steps, kv=kind)
    assert len(calls) == shape.layers * (prompt + steps - 1)
    held = {key: [_held(torch.cat(x, 1), kind) for x in zip(*parts)]
            for key, parts in written.items()}
    for n, (own, shared, tokens, q, out, lse) in enumerate(calls):
        if n % 5 and tokens % page > 2:
            continue  # every fifth call, and those about a page's first tokens
        for row in range(q.shape[0]):
            k, v = (x[row, :tokens] for x in held[own])
            seen = torch.ones((shape.kv_heads, tokens), dtype=torch.bool)
            if shared is not None:
                seen[:shape.local_heads, :max(0, tokens - window)] = False
                pk, pv = (x[0] for x in held[shared])
                assert len(pk) == prompt
                k, v = torch.cat((pk, k)), torch.cat((pv, v))
                seen = torch.cat((torch.ones((shape.kv_heads, prompt), dtype=torch.bool), seen), 1)
            want, want_lse, tol, tol_lse = _reference(
                q[row].double().view(shape.kv_heads, shape.group, -1), k, v, seen)
            got = out[row].view(want.shape)
            assert float((got - want).abs().max()) <= tol, (n, row)
            err = (lse[row].view(want_lse.shape) - want_lse).abs()
            assert bool((err <= tol_lse + want_lse.abs() * U).all()), (n, row)
