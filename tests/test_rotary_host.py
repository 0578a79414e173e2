"""Angles of the rotary positions by their formulas, and refusals of the entry points
before anything is launched (no GPU)."""
import ctypes
import math

import pytest

from paper_2605_20600_amd import binding as B
from test_paged_launch_host import call  # noqa: F401  (a fixture)

FAKE = 0x7F0000000000  # 256-byte aligned, never dereferenced by these calls
I, U = B.HEADKV_ERR_INVALID_ARG, B.HEADKV_ERR_UNSUPPORTED


def _rot(**kw):
    base = dict(head_dim=128, rotary_dims=64, layout=0, axes=1, norm=0, eps=1e-6, scale=1.0,
                scaling=0, original_len=4096, base=10000.0, factor=4.0, low=1.0, high=32.0)
    return B.RotaryConfig(**{**base, **kw})


def _rows(**kw):
    base = dict(in_=FAKE, out=FAKE, in_row=4096, in_token=1024, in_head=128, out_row=4096,
                out_token=1024, out_head=128, weight=None, bias=None, heads=4, per_head=0)
    return B.RotaryRowsArg(**{**base, **kw})


def _cfg(**kw):
    base = dict(kv_type=B.HEADKV_KV_INT8, head_dim=128, kv_heads=4, group=2, page_tokens=64,
                num_pages=100)
    return B.PagedConfig(**{**base, **kw})


def _lists(**kw):
    base = dict(pages=FAKE, len=FAKE, first=None, order=None, lists=3, max_pages=5, extra=0,
                max_len=300)
    return B.PagedListsArg(**{**base, **kw})


def _status(name, *args):
    st = getattr(B.load_paged(), name)(*args)
    assert st == B.HEADKV_OK or B.headkv_last_error() != ""
    return st


def _rotary(cfg=None, turns=FAKE, positions=FAKE, rows=2, tokens=4, counts=None, q=None, k=None):
    return _status("headkv_rotary", cfg or _rot(), turns, positions, rows, tokens, counts,
                   q or _rows(), k, None)


def _write(pcfg=None, pool=FAKE, lists=None, rot=None, turns=FAKE, positions=FAKE, tokens=4,
           counts=None, q=None, k=None, v=FAKE, strides=(4096, 1024, 128)):
    return _status("headkv_paged_write_rotary", pcfg or _cfg(), pool, lists or _lists(),
                   rot or _rot(), turns, positions, tokens, counts, q, k or _rows(), v, *strides,
                   None)


def _close(got, want):
    # 64-bit numbers through a power and a few products: a few units in the last place,
    # times the logarithm that the power takes (20 at most)
    assert len(got) == len(want)
    for a, b in zip(got, want):
        assert abs(a - b) <= 64 * 2.0 ** -53 * abs(b), (a, b)


@pytest.mark.parametrize("axes", (1, 2))
@pytest.mark.parametrize("r", (0, 16, 48, 128))
def test_turns_of_a_position(axes, r):
    n = r // axes
    plain = [10000.0 ** (-2 * (j % (n // 2)) / n) for j in range(r // 2)]
    two_pi = 2 * math.pi
    _close(B.headkv_rotary_plan(_rot(rotary_dims=r, axes=axes)), [w / two_pi for w in plain])
    _close(B.headkv_rotary_plan(_rot(rotary_dims=r, axes=axes, scaling=B.HEADKV_SCALE_LINEAR)),
           [w / 4 / two_pi for w in plain])
    if r:
        got = B.headkv_rotary_plan(_rot(rotary_dims=r, axes=axes, scaling=B.HEADKV_SCALE_BASE))
        # the fastest pair as it was, the slowest as if positions were divided by the factor
        _close([got[0], got[n // 2 - 1]], [plain[0] / two_pi, plain[n // 2 - 1] / 4 / two_pi])
    bands = []
    for w in plain:
        length = two_pi / w
        if length <= 4096 / 32.0:
            bands.append(w)
        elif length >= 4096 / 1.0:
            bands.append(w / 4)
        else:
            t = (4096 / length - 1) / 31
            bands.append(t * w + (1 - t) * w / 4)
    _close(B.headkv_rotary_plan(_rot(rotary_dims=r, axes=axes, scaling=B.HEADKV_SCALE_BANDS)),
           [w / two_pi for w in bands])


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=96), U), (dict(rotary_dims=-16), U), (dict(rotary_dims=24), U),
    (dict(rotary_dims=144), U), (dict(layout=2), I), (dict(axes=0), U), (dict(axes=3), U),
    (dict(norm=3), I), (dict(norm=-1), I), (dict(eps=-1.0), I), (dict(eps=math.nan), I),
    (dict(eps=math.inf), I), (dict(scale=math.inf), I), (dict(scale=math.nan), I)])
def test_configs(kw, status):
    assert _status("headkv_rotary_plan", _rot(**kw), (ctypes.c_double * 64)()) == status
    assert _rotary(_rot(**kw)) == status
    assert _write(rot=_rot(**kw)) == status


@pytest.mark.parametrize("kw", [
    dict(base=0.0), dict(base=-2.0), dict(base=math.nan), dict(scaling=4), dict(scaling=-1),
    dict(scaling=1, factor=0.0), dict(scaling=2, factor=math.inf), dict(scaling=2, factor=1e300),
    dict(scaling=3, low=-1.0), dict(scaling=3, low=32.0), dict(scaling=3, high=math.inf),
    dict(scaling=3, original_len=0), dict(scaling=3, low=math.nan)])
def test_angles_refused(kw):
    kw = {"rotary_dims": 16, "axes": 2, **kw} if kw.get("factor") == 1e300 else kw
    assert _status("headkv_rotary_plan", _rot(**kw), (ctypes.c_double * 64)()) == I


def test_plan_needs_a_place():
    assert _status("headkv_rotary_plan", None, None) == I
    assert _status("headkv_rotary_plan", _rot(), None) == I
    assert _status("headkv_rotary_plan", _rot(rotary_dims=0), None) == B.HEADKV_OK


ROWS = [
    (dict(in_=None), I), (dict(in_=FAKE + 8), I), (dict(in_row=-8), I), (dict(in_token=4), I),
    (dict(in_head=130), I), (dict(weight=FAKE + 4), I), (dict(bias=FAKE + 8), I),
    (dict(heads=-1), U), (dict(heads=65537), U), (dict(per_head=2), I)]


@pytest.mark.parametrize("kw,status", ROWS + [
    (dict(out=None), I), (dict(out=FAKE + 2), I), (dict(out_row=4), I), (dict(out_token=-8), I),
    (dict(out_head=64), I), (dict(out_token=0), I), (dict(out_row=0), I)])
def test_rows_refused(kw, status):
    assert _rotary(q=_rows(**kw)) == status
    assert _rotary(k=_rows(**kw)) == status
    if kw != dict(heads=-1):
        assert _write(q=_rows(**kw)) == status


@pytest.mark.parametrize("kw,status", ROWS + [(dict(heads=0), I), (dict(heads=3), I)])
def test_keys_for_a_cache_refused(kw, status):
    assert _write(k=_rows(**kw)) == status


def test_other_arguments():
    assert _rotary(turns=None) == I
    assert _rotary(positions=None) == I
    assert _rotary(turns=FAKE + 4) == I
    assert _rotary(positions=FAKE + 2) == I
    assert _rotary(counts=FAKE + 2) == I
    assert _rotary(rows=-1) == I
    assert _rotary(tokens=-1) == I
    # nothing to do: no address is needed
    for kw in (dict(rows=0), dict(tokens=0)):
        assert _rotary(turns=None, positions=None, q=_rows(in_=None), **kw) == B.HEADKV_OK
    assert _status("headkv_rotary", _rot(), None, None, 2, 4, None, None, None,
                   None) == B.HEADKV_OK
    assert _write(tokens=0, turns=None, v=None) == B.HEADKV_OK
    assert _write(tokens=-1) == I
    assert _write(pool=None) == I
    assert _write(pool=FAKE + 128) == I
    assert _write(v=None) == I
    assert _write(v=FAKE + 8) == I
    assert _write(strides=(4096, 1028, 128)) == I
    assert _write(pcfg=_cfg(head_dim=64)) == I
    assert _write(lists=_lists(lists=0)) == I
    assert _write(lists=_lists(pages=None)) == I
    assert _write(positions=None) == I
    assert _status("headkv_paged_write_rotary", _cfg(), FAKE, _lists(), _rot(), FAKE, FAKE, 1,
                   None, None, None, FAKE, 0, 0, 0, None) == I


ROWS_ARG = "B.RotaryRowsArg(FAKE, FAKE, 128, 128, 128, 128, 128, 128, None, None, {heads}, 0)"


def test_grids(call):  # noqa: F811
    rot = "B.RotaryConfig({d}, 64, 0, 1, 0, 0, 1, 0, 0, 1, 0, 0, 0)"
    run = "L.headkv_rotary(" + rot + ", FAKE, FAKE, {rows}, {tokens}, None, " + ROWS_ARG + ", None, None)"
    # a token's heads among as many wavefronts as there are steps of 8, or as fill the card
    for rows, tokens, heads, waves in ((1, 1, 1, 1), (8, 1, 64, 64), (8, 1, 65, 72),
                                       (100, 100, 64, 10000)):
        st, got = call(run.format(d=128, rows=rows, tokens=tokens, heads=heads))
        assert st == B.HEADKV_OK and got == [((waves + 3) // 4, 256)], got
    st, got = call(run.format(d=64, rows=1 << 12, tokens=1 << 13, heads=1))
    assert st == B.HEADKV_OK and got[0][0] * got[0][1] < 1 << 32
    st, got = call(run.format(d=64, rows=1 << 14, tokens=1 << 13, heads=1))
    assert st == U and not got
    write = ("L.headkv_paged_write_rotary(cfg(head_dim={d}, kv_heads={heads}), FAKE, lists({rows}), "
             + rot + ", FAKE, FAKE, {tokens}, None, None, " + ROWS_ARG + ", FAKE, 128, 128, 128, None)")
    for d in (64, 128):
        for tokens in (1, 4, 5):  # as many lists as there may be
            st, got = call(write.format(d=d, rows=1 << 14, heads=1024, tokens=tokens))
            assert st == B.HEADKV_OK and len(got) == 1 and got[0][0] * got[0][1] < 1 << 32
