"""Grids of the paged calls at their limits (no GPU): libheadkv.so over
tests/host/fake_launch.cpp, which notes launches instead of making them."""
import os
import subprocess
import sys

import pytest

from paper_2605_20600_amd import binding as B
from paper_2605_20600_amd.build import ROOT

HERE = os.path.dirname(os.path.abspath(__file__))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
U = B.HEADKV_ERR_UNSUPPORTED

RUN = """
import ctypes, sys
fake = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
from paper_2605_20600_amd import binding as B
FAKE = 0x7F0000000000
L = B.load_paged()

def cfg(**kw):
    base = dict(kv_type=B.HEADKV_KV_INT8, head_dim=64, kv_heads=1, group=1, page_tokens=256,
                num_pages=100)
    return B.PagedConfig(**{**base, **kw})

def lists(n, max_pages=1, max_len=256):
    return B.PagedListsArg(FAKE, FAKE, None, None, n, max_pages, 0, max_len)

def attn(c, own, shared):
    return L.headkv_paged_attn(c, FAKE, own, shared, FAKE, FAKE, 0, FAKE, None, FAKE, 1 << 62, None)

def write(c, n, tokens):
    return L.headkv_paged_write(c, FAKE, lists(n), FAKE, FAKE, 0, 0, 0, tokens, None, None)

def read(c, tokens, n=1):
    return L.headkv_paged_read(c, FAKE, lists(n), 0, tokens, FAKE, FAKE, 128, 128, 128, None)

print(eval(sys.argv[2]))
for i in range(fake.fake_launches()):
    g, b = ctypes.c_uint(), ctypes.c_uint()
    fake.fake_launch(i, ctypes.byref(g), ctypes.byref(b))
    print(g.value, b.value)
"""


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    lib = tmp_path_factory.mktemp("fake") / "fake_launch.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-I",
                    os.path.join(ROCM, "include"), os.path.join(HERE, "host", "fake_launch.cpp"),
                    "-o", str(lib)], check=True)

    def run(expr):
        """The call's status, and (blocks, threads of one) of its launches."""
        out = subprocess.run([sys.executable, "-c", RUN, str(lib), expr], check=True, cwd=ROOT,
                             stdout=subprocess.PIPE, text=True).stdout.split()
        n = [int(x) for x in out]
        return n[0], list(zip(n[1::2], n[2::2]))
    return run


def test_few_and_many(call):
    # that launches are seen at all: 3 own lists, then with a prefix of two chunks
    st, got = call("attn(cfg(), lists(3), lists(1, 2, 512))")
    assert st == B.HEADKV_OK and len(got) == 1 and got[0] == (5, 256)
    st, got = call("write(cfg(), 3, 9)")
    assert st == B.HEADKV_OK and got == [(1, 256)]


# Blocks of the prefixes, by chunks and tiles of columns, and of own lists (four short
# ones to a block): 2^24 and 2^23 prefixes of a chunk, the latter also beside own lists
# that take 2^23 blocks; then blocks of 512 threads for many columns.
@pytest.mark.parametrize("expr,shared,own", (
    ("attn(cfg(kv_heads=1024), lists(1), lists(1 << 14))", 1 << 24, 1 << 10),
    ("attn(cfg(kv_heads=1024), lists(64), lists(1 << 13))", 1 << 23, 1 << 14),
    ("attn(cfg(kv_heads=1024), lists(64, 512, 1 << 17), lists(1 << 13))", 1 << 23, 1 << 23),
    ("attn(cfg(kv_heads=4, group=16), lists(1 << 17), lists(1, 1 << 12, 1 << 20))", 1 << 24, 1 << 17),
    ("attn(cfg(kv_heads=4, group=16), lists(1 << 18), lists(1, 1 << 13, 1 << 21))", 1 << 26, 1 << 18),
    ("attn(cfg(kv_heads=64, group=16), lists(1 << 17), lists(1, 1 << 8, 1 << 16))", 1 << 24, 1 << 21),
))
def test_shared_prefixes_of_any_number(call, expr, shared, own):
    st, got = call(expr)
    assert st == B.HEADKV_OK
    assert all(g * b < 1 << 32 for g, b in got), got
    assert sum(g for g, _ in got) == shared + own, got


def test_shared_prefixes_past_the_limit(call):
    st, got = call("attn(cfg(kv_heads=64, group=16), lists(1 << 18), lists(1 << 18, 1 << 20, 1 << 28))")
    assert st == U and not got


@pytest.mark.parametrize("d", (64, 128))
def test_tokens_of_as_many_lists_as_there_may_be(call, d):
    for tokens in (1, 4, 5):
        st, got = call(f"write(cfg(head_dim={d}, kv_heads=1024), 1 << 14, {tokens})")
        assert st == B.HEADKV_OK and len(got) == 1 and got[0][0] * got[0][1] < 1 << 32
    st, got = call(f"write(cfg(head_dim={d}), 1, (1 << 28) - 64)")
    assert st == B.HEADKV_OK and got[0][0] * got[0][1] < 1 << 32


@pytest.mark.parametrize("d", (64, 128))
def test_too_many_tokens_for_a_call(call, d):
    for expr in ("write(cfg(head_dim={d}), 1, (1 << 31) - 1)", "read(cfg(head_dim={d}), (1 << 31) - 1)",
                 "write(cfg(head_dim={d}, kv_heads=1024), 1 << 14, 64)"):
        st, got = call(expr.format(d=d))
        assert st == U and not got


# Sizes at which one kind was measured faster than the other, or as fast: a wavefront for
# a list (blocks of four lists), or a block.
@pytest.mark.parametrize("lists,most,single", (
    (1024, 64, True), (1024, 128, False), (512, 32, False), (512, 64, False), (256, 8, False),
    (2048, 128, True), (2048, 256, False), (4096, 512, True), (12288, 128, True),
    (4096, 1024, False)))
def test_many_short_lists(call, lists, most, single):
    st, got = call(f"L.headkv_paged_attn(cfg(), FAKE, lists({lists}, 16, {most}), None, None, FAKE, 0, "
                   "FAKE, None, FAKE, 1 << 62, None)")
    assert st == B.HEADKV_OK and got == [(lists // 4 if single else lists, 256)]


# Sizes at which blocks of 512 threads, for 256 columns, were measured faster than tiles of
# 16 columns, or slower.
@pytest.mark.parametrize("kind,heads,group,rows,prefixes,tokens,wide", (
    ("FP4", 8, 4, 64, 1, 16384, False), ("FP4", 8, 4, 96, 1, 16384, False),
    ("FP4", 8, 4, 128, 2, 16384, True), ("FP4", 8, 4, 128, 1, 16384, True),
    ("FP4", 32, 1, 96, 1, 16384, False), ("FP4", 32, 1, 256, 1, 8192, True),
    ("INT8", 8, 4, 32, 1, 16384, False), ("INT8", 8, 4, 48, 1, 16384, False),
    ("INT8", 32, 4, 128, 1, 2048, True), ("INT8", 32, 1, 192, 1, 8192, True),
    ("INT8", 32, 1, 96, 1, 16384, True), ("INT8", 32, 1, 128, 1, 8192, False),
    ("INT8", 8, 4, 64, 1, 2048, False),
    ("BF16", 8, 4, 24, 1, 16384, True), ("BF16", 8, 4, 32, 1, 16384, True),
    ("BF16", 32, 1, 96, 1, 2048, False), ("BF16", 32, 1, 96, 1, 8192, True)))
def test_prefixes_of_many_columns(call, kind, heads, group, rows, prefixes, tokens, wide):
    st, got = call(f"attn(cfg(kv_type=B.HEADKV_KV_{kind}, head_dim=128, kv_heads={heads}, "
                   f"group={group}), lists({rows}), lists({prefixes}, 64, {tokens}))")
    assert st == B.HEADKV_OK and (512 in [b for _, b in got]) == wide, got


@pytest.mark.parametrize("kind", ("BF16", "INT8", "FP4"))
@pytest.mark.parametrize("rows,heads,group", ((256, 8, 1), (64, 8, 4), (40, 32, 4), (16, 2, 16), (12, 20, 13)))
def test_workspaces_hold_every_shorter_prefix(kind, rows, heads, group):
    # also where a longer prefix goes to the other kind of blocks
    cfg = B.PagedConfig(getattr(B, f"HEADKV_KV_{kind}"), 128, heads, group, 64, 100)
    for prefixes in (1, 2):
        last = 0
        for n in range(0, 40000, 32):
            need = B.headkv_paged_attn_plan(cfg, B.PagedListsArg(None, None, None, None, rows, 9, 0, 576),
                                            B.PagedListsArg(None, None, None, None, prefixes, 1000, 0, n))
            assert need >= last, n
            last = need
