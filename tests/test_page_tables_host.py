"""Refusals of the page tables' entry points before anything is launched, and their grids
at the limits (no GPU)."""
import ctypes

import pytest

from paper_2605_20600_amd import binding as B
from test_paged_launch_host import call  # noqa: F401  (a fixture)

FAKE = 0x7F0000000000  # 256-byte aligned, never dereferenced by these calls
I, U, C = B.HEADKV_ERR_INVALID_ARG, B.HEADKV_ERR_UNSUPPORTED, B.HEADKV_ERR_CAPACITY


def _tables(**kw):
    base = dict(pages=FAKE, len=FAKE, first=FAKE, order=None, window=None, free_pages=FAKE,
                free_state=FAKE, kv_heads=4, page_tokens=64, num_pages=100, lists=6, rows=3,
                max_pages=5)
    return B.PagedTablesArg(**{**base, **kw})


def _extend(t=None, advance=None, counts=None, tokens=1, ws=FAKE, size=1 << 20):
    st = B.load_paged().headkv_paged_extend(t, advance, counts, tokens, ws, size, None)
    assert st == B.HEADKV_OK or B.headkv_last_error() != ""
    return st


@pytest.mark.parametrize("kw,status", [
    (dict(kv_heads=0), U), (dict(kv_heads=1025), U), (dict(page_tokens=48), U),
    (dict(num_pages=0), I), (dict(lists=0), I), (dict(rows=0), I), (dict(rows=4), I),
    (dict(max_pages=0), I), (dict(lists=3 << 21, max_pages=1), U),
    (dict(max_pages=(1 << 22) + 1, lists=3), U), (dict(lists=3 << 10, max_pages=1 << 19), U)])
def test_sizes(kw, status):
    size = ctypes.c_size_t()
    assert B.load_paged().headkv_paged_extend_plan(_tables(**kw), size) == status
    assert _extend(_tables(**kw)) == status


@pytest.mark.parametrize("name", ("pages", "len", "first", "free_pages", "free_state"))
def test_arrays(name):
    assert _extend(_tables(**{name: None})) == I
    assert _extend(_tables(**{name: FAKE + 2})) == I


def test_other_arguments():
    assert _extend(None) == I
    assert B.load_paged().headkv_paged_extend_plan(_tables(), None) == I
    for kw in (dict(t=_tables(order=FAKE + 1)), dict(t=_tables(window=FAKE + 2)),
               dict(advance=FAKE + 2), dict(counts=FAKE + 1), dict(tokens=-1), dict(ws=None),
               dict(ws=FAKE + 64)):
        assert _extend(**{"t": _tables(), **kw}) == I
    assert _extend(_tables(), tokens=(1 << 24) + 1) == U
    assert _extend(_tables(), size=8) == C


def test_grids(call):  # noqa: F811
    arg = ("B.PagedTablesArg(FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, {heads}, 64, 100, {lists}, "
           "{rows}, 1)")
    run = "L.headkv_paged_extend(" + arg + ", None, None, 1, FAKE, 1 << 20, None)"
    st, got = call(run.format(heads=32, lists=8, rows=8))  # in one launch
    assert st == B.HEADKV_OK and got == [(1, 1024)]
    for heads, lists, rows in ((1024, 1 << 14, 1 << 14), (1, 1 << 24, 1), (3, 5000, 100)):
        st, got = call(run.format(heads=heads, lists=lists, rows=rows))
        assert st == B.HEADKV_OK and len(got) == 3
        assert all(b == 1024 and g * b < 1 << 32 for g, b in got)
        assert got[0] == got[1] and got[0][0] <= 512  # counts that a block adds up
        assert got[2][0] == got[0][0] + min(lists // rows, 4096)
