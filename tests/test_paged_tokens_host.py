"""Refusals of the attention of several tokens before anything is launched, and its grids
at their limits (no GPU)."""
import ctypes

import pytest

from paper_2605_20600_amd import binding as B
from test_paged_host import _cfg, _lists
from test_paged_launch_host import call  # noqa: F401  (a fixture)

FAKE = 0x7F0000000000  # 256-byte aligned, never dereferenced by these calls
I, U, C = B.HEADKV_ERR_INVALID_ARG, B.HEADKV_ERR_UNSUPPORTED, B.HEADKV_ERR_CAPACITY


def _attn(cfg=None, pool=FAKE, own=None, shared=None, share=None, tokens=5, counts=None,
          window=None, q=FAKE, strides=(5120, 1024), out=FAKE, lse=None, ws=FAKE, size=1 << 30):
    st = B.load_paged().headkv_paged_attn_tokens(
        cfg or _cfg(), pool, own or _lists(), shared, share, tokens, counts, window, q, *strides,
        out, lse, ws, size, None)
    assert st == B.HEADKV_OK or B.headkv_last_error() != ""
    return st


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=_cfg(head_dim=96)), U), (dict(own=_lists(pages=None)), I), (dict(pool=None), I),
    (dict(pool=FAKE + 16), I), (dict(shared=_lists()), I), (dict(share=FAKE), I),
    (dict(shared=_lists(lists=0), share=FAKE), I), (dict(shared=_lists(), share=FAKE + 2), I),
    (dict(tokens=-1), I), (dict(counts=FAKE + 2), I), (dict(window=FAKE + 1), I),
    (dict(q=None), I), (dict(q=FAKE + 8), I), (dict(strides=(-8, 1024)), I),
    (dict(strides=(5120, 12)), I), (dict(out=None), I), (dict(out=FAKE + 8), I),
    (dict(lse=FAKE + 2), I), (dict(ws=None), I), (dict(ws=FAKE + 8), I), (dict(size=100), C),
    (dict(own=_lists(lists=1 << 21), tokens=20), U), (dict(tokens=2 ** 31 - 1), U)])
def test_refusals(kw, status):
    assert _attn(**kw) == status


def test_nothing_to_do():
    assert _attn(tokens=0, q=None, out=None, ws=None, size=0) == B.HEADKV_OK


def test_plan():
    size = ctypes.c_size_t()
    plan = B.load_paged().headkv_paged_attn_tokens_plan
    assert plan(_cfg(), _lists(), None, -1, size) == I
    assert plan(_cfg(), _lists(), None, 1, None) == I
    assert plan(_cfg(), _lists(lists=1 << 21), None, 20, size) == U


@pytest.mark.parametrize("kind", ("BF16", "INT8", "FP4"))
@pytest.mark.parametrize("rows,heads,group,tokens", (
    (3, 4, 2, 9), (1, 1, 1, 17), (1, 8, 4, 8), (4, 8, 4, 256), (40, 32, 1, 5), (512, 32, 1, 3),
    (300, 32, 4, 64), (2000, 8, 1, 1), (1, 2, 16, 500)))
@pytest.mark.parametrize("shared", (False, True))
def test_workspaces_hold_every_shorter_length(kind, rows, heads, group, tokens, shared):
    # also where longer lists go to the other kind of blocks, and in what a launch asks for
    cfg = _cfg(kv_type=getattr(B, f"HEADKV_KV_{kind}"), kv_heads=heads, group=group)
    more = _lists(lists=2, max_len=2000, max_pages=40) if shared else None
    last = 0
    for n in list(range(0, 4200, 60)) + list(range(4200, 140000, 1777)):
        own = _lists(lists=rows, max_pages=1 << 12, max_len=n)
        need = B.headkv_paged_attn_tokens_plan(cfg, own, more, tokens)
        assert need >= last, n
        last = need
    # what lists of many rows take does not grow with their length
    if rows * heads * tokens >= 1 << 14 and not shared:
        assert last < 1 << 31


def test_grids(call):  # noqa: F811
    run = ("L.headkv_paged_attn_tokens(cfg(kv_heads={heads}, group={group}), FAKE, lists({rows}, 16, "
           "{most}), None, None, {tokens}, None, None, FAKE, 0, 0, FAKE, None, FAKE, 1 << 62, None)")
    # 16 / group tokens to a cut
    for rows, heads, group, tokens, cuts in ((3, 2, 1, 16, 1), (3, 2, 1, 17, 2), (3, 2, 3, 5, 1),
                                             (3, 2, 3, 6, 2), (3, 2, 16, 3, 3)):
        st, got = call(run.format(rows=rows, heads=heads, group=group, tokens=tokens, most=100))
        assert st == B.HEADKV_OK and got == [(rows * heads * cuts, 256)], got
    # 128 / group of them, in blocks of 512 threads, where there is work for them
    for rows, heads, group, tokens, cuts in ((300, 2, 4, 64, 2), (300, 2, 4, 65, 3),
                                             (300, 2, 3, 86, 3), (300, 2, 16, 16, 2)):
        st, got = call(run.format(rows=rows, heads=heads, group=group, tokens=tokens, most=200))
        assert st == B.HEADKV_OK and got == [(rows * heads * cuts, 512)], got
    # few cuts: one block for each CU at most, and the sum of parts
    st, got = call(run.format(rows=4, heads=8, group=4, tokens=256, most=3000))
    assert st == B.HEADKV_OK and got[0] == (256, 512) and got[1][1] == 256 and len(got) == 2, got
    st, got = call(run.format(rows=1 << 14, heads=1024, group=16, tokens=1, most=4000))
    assert st == B.HEADKV_OK and all(g * b < 1 << 32 for g, b in got)


@pytest.mark.parametrize("kind,heads,group,tokens,most", (
    ("BF16", 2, 4, 3, 8192), ("INT8", 2, 8, 2, 16384), ("FP4", 4, 16, 1, 16384)))
def test_blocks_of_256_columns(call, kind, heads, group, tokens, most):  # noqa: F811
    st, got = call(f"L.headkv_paged_attn_tokens(cfg(kv_type=B.HEADKV_KV_{kind}, head_dim=128, "
                   f"kv_heads={heads}, group={group}), FAKE, lists(65, 1, 40), lists(1, 64, {most}), "
                   f"FAKE, {tokens}, None, None, FAKE, 0, 0, FAKE, None, FAKE, 1 << 62, None)")
    assert st == B.HEADKV_OK and 512 in [b for _, b in got], got
