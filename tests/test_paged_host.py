"""Refusals of the paged cache's, its attention's and the token scores' entry
points: the documented status before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2605_20600_amd import binding as B

FAKE = 0x7F0000000000  # 256-byte aligned, never dereferenced by these calls
I, U, C = B.HEADKV_ERR_INVALID_ARG, B.HEADKV_ERR_UNSUPPORTED, B.HEADKV_ERR_CAPACITY
S64 = ctypes.c_int64


def _cfg(**kw):
    base = dict(kv_type=B.HEADKV_KV_INT8, head_dim=128, kv_heads=4, group=2, page_tokens=64,
                num_pages=100)
    return B.PagedConfig(**{**base, **kw})


def _lists(**kw):
    base = dict(pages=FAKE, len=FAKE, first=None, order=None, lists=3, max_pages=5, extra=0, max_len=300)
    return B.PagedListsArg(**{**base, **kw})


def _status(name, *args):
    st = getattr(B.load_paged(), name)(*args)
    assert st == B.HEADKV_OK or B.headkv_last_error() != ""
    return st


@pytest.mark.parametrize("kw,status", [
    (dict(kv_type=3), I), (dict(kv_type=-1), I), (dict(head_dim=96), U), (dict(kv_heads=0), U),
    (dict(kv_heads=1025), U), (dict(group=0), U), (dict(group=17), U), (dict(page_tokens=16), U),
    (dict(page_tokens=96), U), (dict(page_tokens=512), U), (dict(num_pages=0), I)])
def test_config(kw, status):
    assert _status("headkv_paged_plan", _cfg(**kw), None, None) == status
    assert _status("headkv_paged_write", _cfg(**kw), FAKE, _lists(), FAKE, FAKE, 512, 512, 128, 1,
                   None, None) == status
    assert _status("headkv_paged_attn", _cfg(**kw), FAKE, _lists(), None, None, FAKE, 1024, FAKE,
                   None, FAKE, 1 << 30, None) == status


def test_plan():
    # K and V codes, and two scales of two bytes per token
    assert B.headkv_paged_plan(_cfg()) == (64 * (2 * 128 + 4), 100 * 64 * 260)
    assert B.headkv_paged_plan(_cfg(kv_type=B.HEADKV_KV_FP4))[0] == 64 * 2 * (64 + 4)
    assert B.headkv_paged_plan(_cfg(kv_type=B.HEADKV_KV_BF16))[0] == 64 * 2 * 256
    # a whole number of 128 bytes
    assert B.headkv_paged_plan(_cfg(kv_type=B.HEADKV_KV_FP4, head_dim=64, page_tokens=32))[0] == 2176
    big = _cfg(num_pages=2 ** 31 - 1)
    assert B.headkv_paged_plan(big)[1] == 64 * 260 * (2 ** 31 - 1)
    assert _status("headkv_paged_plan", None, None, None) == I


@pytest.mark.parametrize("kw,status", [
    (dict(pages=None), I), (dict(pages=FAKE + 2), I), (dict(len=FAKE + 1), I), (dict(lists=0), I),
    (dict(first=FAKE + 2), I), (dict(order=FAKE + 2), I), (dict(max_pages=0), I), (dict(extra=-1), I), (dict(max_len=-1), I),
    (dict(lists=1 << 24), U), (dict(max_pages=(1 << 22) + 1), U)])
def test_lists(kw, status):
    l = _lists(**kw)
    assert _status("headkv_paged_write", _cfg(), FAKE, l, FAKE, FAKE, 512, 512, 128, 1, None,
                   None) == status
    assert _status("headkv_paged_read", _cfg(), FAKE, l, 0, 1, FAKE, FAKE, 512, 512, 128,
                   None) == status
    assert _status("headkv_paged_attn", _cfg(), FAKE, l, None, None, FAKE, 1024, FAKE, None, FAKE,
                   1 << 40, None) == status
    assert _status("headkv_paged_attn", _cfg(), FAKE, _lists(), l, FAKE, FAKE, 1024, FAKE, None,
                   FAKE, 1 << 40, None) == status


@pytest.mark.parametrize("args", [
    (None, FAKE, FAKE, 512, 512, 128, 1, None), (FAKE + 64, FAKE, FAKE, 512, 512, 128, 1, None),
    (FAKE, None, FAKE, 512, 512, 128, 1, None), (FAKE, FAKE, None, 512, 512, 128, 1, None),
    (FAKE, FAKE + 8, FAKE, 512, 512, 128, 1, None), (FAKE, FAKE, FAKE + 4, 512, 512, 128, 1, None),
    (FAKE, FAKE, FAKE, 516, 512, 128, 1, None), (FAKE, FAKE, FAKE, 512, -8, 128, 1, None),
    (FAKE, FAKE, FAKE, 512, 512, 127, 1, None), (FAKE, FAKE, FAKE, 512, 512, 128, -1, None),
    (FAKE, FAKE, FAKE, 512, 512, 128, 1, FAKE + 2)])
def test_write(args):
    pool, k, v, ls, ts, hs, tokens, counts = args
    assert _status("headkv_paged_write", _cfg(), pool, _lists(), k, v, ls, ts, hs, tokens, counts,
                   None) == I


def test_nothing_to_write_or_read():
    assert _status("headkv_paged_write", _cfg(), FAKE, _lists(), FAKE, FAKE, 512, 512, 128, 0, None,
                   None) == B.HEADKV_OK
    assert _status("headkv_paged_read", _cfg(), FAKE, _lists(), 0, 0, FAKE, FAKE, 512, 512, 128,
                   None) == B.HEADKV_OK


def test_rows_of_no_tokens_need_no_address():
    assert _status("headkv_paged_write", _cfg(), FAKE, _lists(), None, None, 0, 0, 128, 0, None,
                   None) == B.HEADKV_OK
    assert _status("headkv_paged_read", _cfg(), FAKE, _lists(), 0, 0, None, None, 0, 0, 128,
                   None) == B.HEADKV_OK


@pytest.mark.parametrize("strides,tokens", [((64, 512, 128), 1), ((512, 64, 128), 2),
                                            ((512, 512, 0), 1)])
def test_read_refuses_overlapping_rows(strides, tokens):
    assert _status("headkv_paged_read", _cfg(), FAKE, _lists(), 0, tokens, FAKE, FAKE, *strides,
                   None) == I


def test_attention():
    def status(pool=FAKE, own=None, shared=None, share=None, q=FAKE, stride=1024, out=FAKE,
               lse=None, ws=FAKE, size=1 << 40):
        return _status("headkv_paged_attn", _cfg(), pool, own or _lists(), shared, share, q, stride,
                       out, lse, ws, size, None)
    assert status(pool=None) == I and status(pool=FAKE + 128) == I
    assert status(q=None) == I and status(q=FAKE + 8) == I
    assert status(out=None) == I and status(out=FAKE + 4) == I
    assert status(lse=FAKE + 2) == I
    assert status(stride=1023) == I and status(stride=-8) == I
    assert status(shared=_lists()) == I and status(share=FAKE) == I
    assert status(shared=_lists(), share=FAKE + 2) == I
    need = B.headkv_paged_attn_plan(_cfg(), _lists(), _lists(max_len=10 ** 6, max_pages=10 ** 5))
    if need:
        assert status(shared=_lists(max_len=10 ** 6, max_pages=10 ** 5), share=FAKE,
                      size=need - 1) == C
        assert status(shared=_lists(max_len=10 ** 6, max_pages=10 ** 5), share=FAKE, ws=None) == I
        assert status(shared=_lists(max_len=10 ** 6, max_pages=10 ** 5), share=FAKE,
                      ws=FAKE + 64) == I


def test_attention_workspace_does_not_shrink():
    for shared in (None, 1, 7000):
        last = 0
        for n in (0, 1, 31, 64, 65, 500, 1000, 4096, 5000, 100000):
            s = None if shared is None else _lists(lists=2, max_pages=200, max_len=shared)
            need = B.headkv_paged_attn_plan(_cfg(), _lists(max_pages=2000, max_len=n), s)
            assert need >= last, (shared, n)
            last = need


@pytest.mark.parametrize("lists,heads", ((20, 5), (1, 1), (3, 4), (8, 8), (64, 32)))
@pytest.mark.parametrize("kind", (B.HEADKV_KV_BF16, B.HEADKV_KV_INT8, B.HEADKV_KV_FP4))
def test_attention_workspace_holds_every_shorter_length(lists, heads, kind):
    cfg, lists2 = _cfg(kv_heads=heads, kv_type=kind), max(1, lists // 8)
    own = shared = 0
    for n in range(0, 40000, 32):
        a = _lists(lists=lists, max_pages=1000, max_len=n)
        b = _lists(lists=lists2, max_pages=1000, max_len=n)
        need = B.headkv_paged_attn_plan(cfg, a, None)
        assert need >= own, n
        own = need
        need = B.headkv_paged_attn_plan(cfg, _lists(lists=lists, max_pages=1, max_len=1), b)
        assert need >= shared, n
        shared = need


def test_scores():
    def status(logits=FAKE, kind=B.HEADKV_LOGITS_BF16, rows=4, vocab=100, stride=100, tokens=FAKE,
               temperature=1.0, top=5, logprob=FAKE, entropy=None, rank=None, tv=FAKE, ti=FAKE,
               ws=FAKE, size=1 << 40):
        return _status("headkv_token_logprobs", logits, kind, rows, vocab, S64(stride), tokens,
                       temperature, top, logprob, entropy, rank, tv, ti, ws, size, None)
    assert status(rows=-1) == I and status(vocab=0) == I and status(vocab=(1 << 24) + 1) == U
    assert status(kind=2) == I and status(stride=99) == I
    assert status(top=-1) == I and status(top=33) == I and status(top=5, vocab=4, stride=4) == I
    assert status(temperature=0.0) == I and status(temperature=-1.0) == I
    assert status(temperature=float("nan")) == I and status(temperature=float("inf")) == I
    assert status(temperature=1e-45) == I  # its inverse overflows
    assert status(logits=None) == I and status(tokens=None) == I and status(logprob=None) == I
    assert status(tv=None) == I and status(ti=None) == I
    assert status(logits=FAKE + 1) == I
    assert status(logits=FAKE + 2, kind=B.HEADKV_LOGITS_F32) == I
    assert status(tokens=FAKE + 2) == I and status(entropy=FAKE + 2) == I
    assert status(rows=0) == B.HEADKV_OK
    need = B.headkv_logprobs_plan(8, 1 << 20, 32)
    if need:
        kw = dict(rows=8, vocab=1 << 20, stride=1 << 20, top=32)
        assert status(size=need - 1, **kw) == C
        assert status(ws=None, **kw) == I and status(ws=FAKE + 64, **kw) == I


def test_scores_workspace_does_not_shrink():
    sizes = [B.headkv_logprobs_plan(r, v, t) for r in (1, 3, 100, 5000)
             for v in (1000, 16384, 65536, 200000) for t in (0, 1, 32)]
    grid = iter(sizes)
    got = {(r, v, t): next(grid) for r in (1, 3, 100, 5000)
           for v in (1000, 16384, 65536, 200000) for t in (0, 1, 32)}
    for (r, v, t), n in got.items():
        for (r2, v2, t2), n2 in got.items():
            if r2 >= r and v2 >= v and t2 >= t:
                assert n2 >= n, ((r, v, t), (r2, v2, t2))
