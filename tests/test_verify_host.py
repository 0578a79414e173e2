"""Refusals of the verification of drafted tokens before anything is launched, and its
workspace (no GPU)."""
import ctypes
import math

import pytest

from paper_2605_20600_amd import binding as B

FAKE = 0x7F0000000000  # 256-byte aligned, never dereferenced by these calls
I, U, C = B.HEADKV_ERR_INVALID_ARG, B.HEADKV_ERR_UNSUPPORTED, B.HEADKV_ERR_CAPACITY


def _verify(logits=FAKE, draft=FAKE, kind=B.HEADKV_LOGITS_BF16, rows=2, drafts=3, vocab=100,
            strides=(400, 100, 300, 100), tokens=FAKE, counts=None, uniforms=FAKE, t=1.0,
            out=FAKE, count=FAKE, logprob=None, ws=FAKE, size=1 << 30):
    st = B.load_paged().headkv_verify_drafts(logits, draft, kind, rows, drafts, vocab, *strides,
                                             tokens, counts, uniforms, t, out, count, logprob, ws,
                                             size, None)
    assert st == B.HEADKV_OK or B.headkv_last_error() != ""
    return st


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), I), (dict(logits=FAKE + 1), I), (dict(draft=FAKE + 1), I),
    (dict(kind=B.HEADKV_LOGITS_F32, logits=FAKE + 2), I), (dict(kind=2), I), (dict(rows=-1), I),
    (dict(drafts=-1), U), (dict(drafts=64), U), (dict(vocab=0), I), (dict(vocab=(1 << 24) + 1), U),
    (dict(strides=(-1, 100, 300, 100)), I), (dict(strides=(400, 100, 300, -1)), I),
    (dict(tokens=None), I), (dict(tokens=FAKE + 2), I), (dict(counts=FAKE + 2), I),
    (dict(uniforms=None), I), (dict(uniforms=FAKE + 2), I), (dict(t=-1.0), I),
    (dict(t=math.nan), I), (dict(t=math.inf), I), (dict(t=5e-309), I), (dict(out=None), I),
    (dict(out=FAKE + 2), I), (dict(count=None), I), (dict(count=FAKE + 1), I),
    (dict(logprob=FAKE + 2), I), (dict(ws=None), I), (dict(ws=FAKE + 128), I), (dict(size=0), C)])
def test_refusals(kw, status):
    assert _verify(**kw) == status


def test_nothing_to_do():
    assert _verify(rows=0, logits=None, uniforms=None, out=None, count=None, ws=None,
                   size=0) == B.HEADKV_OK


def test_workspace_grows():
    size = ctypes.c_size_t()
    assert B.load_paged().headkv_verify_plan(1, 1, 1, None) == I
    assert B.load_paged().headkv_verify_plan(1, 64, 1, size) == U
    last = 0
    for rows, drafts, vocab in ((0, 0, 1), (1, 0, 1), (1, 4, 1), (1, 4, 16384), (8, 4, 16384),
                                (8, 63, 16384), (8, 63, 1 << 24), (300, 63, 1 << 24)):
        need = B.headkv_verify_plan(rows, drafts, vocab)
        assert need >= last and need % 8 == 0
        last = need
    # calls of many rows take turns in the same places
    assert B.headkv_verify_plan(1 << 20, 4, 1000) == B.headkv_verify_plan(1 << 16, 4, 1000)
