"""Host-only checks of nt_op_attn_prompt, nt_op_attn_tree, nt_op_kv_resize and nt_op_kv_keep: what they
refuse, with which status, and workspace sizes.  The pointers are never read."""
import ctypes
import re

import pytest

from tests.test_paged_cpu import P, _cache, nt   # noqa: F401  (the fixture)


def prompt(nt, **kw):
    a = dict(dtype=1, q=P, q_ld=512, n_heads=4, k=P, v=P, kv_ld=512, n_kv_heads=2, d_head=64, off=P, n_seqs=0, n_rows=0,
             causal=1, scale=0.125, out=P, out_ld=256)
    a.update(kw)
    return nt.load_library().nt_op_attn_prompt(a["dtype"], a["q"], a["q_ld"], a["n_heads"], a["k"], a["v"], a["kv_ld"],
                                               a["n_kv_heads"], a["d_head"], a["off"], a["n_seqs"], a["n_rows"],
                                               a["causal"], a["scale"], a["out"], a["out_ld"], None)


def tree(nt, cache=None, **kw):
    c = _cache(nt) if cache is None else cache
    a = dict(q=P, q_ld=256, n_heads=4, off=P, mask=P, lens=P, n_seqs=0, n_rows=0, max_new=8, max_len=64, scale=0.125, out=P,
             out_ld=256, ws=None, ws_bytes=0)
    a.update(kw)
    return nt.load_library().nt_op_attn_tree(ctypes.byref(c) if c else None, a["q"], a["q_ld"], a["n_heads"], a["off"],
                                             a["mask"], a["lens"], a["n_seqs"], a["n_rows"], a["max_new"], a["max_len"],
                                             a["scale"], a["out"], a["out_ld"], a["ws"], a["ws_bytes"], None)


def resize(nt, **kw):
    a = dict(page_len=16, n_pages=8, max_pages=4, table=P, lens=P, add=P, n_seqs=3, ring=P, state=P, off=P, pos=P, slot=P,
             max_rows=9)
    a.update(kw)
    return nt.load_library().nt_op_kv_resize(a["page_len"], a["n_pages"], a["max_pages"], a["table"], a["lens"], a["add"],
                                             a["n_seqs"], a["ring"], a["state"], a["off"], a["pos"], a["slot"],
                                             a["max_rows"], None)


def keep(nt, cache=None, **kw):
    c = _cache(nt) if cache is None else cache
    a = dict(off=P, lens=P, path=P, max_path=4, n_path=P, n_seqs=0, add=P)
    a.update(kw)
    return nt.load_library().nt_op_kv_keep(ctypes.byref(c) if c else None, a["off"], a["lens"], a["path"], a["max_path"],
                                           a["n_path"], a["n_seqs"], a["add"], None)


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("kw", [
    {"dtype": 3}, {"dtype": -1}, {"q": None}, {"k": None}, {"v": None}, {"off": None}, {"out": None}, {"d_head": 48},
    {"d_head": 256}, {"n_kv_heads": 0}, {"n_kv_heads": 3}, {"n_heads": 0}, {"n_heads": 5}, {"n_seqs": -1}, {"n_rows": -1},
    {"q_ld": 255}, {"kv_ld": 127}, {"out_ld": 248}, {"q_ld": 260}, {"kv_ld": 130}, {"out_ld": 258}, {"q": P + 8}, {"k": P + 2},
    {"v": P + 4}, {"out": P + 8}, {"scale": INF}, {"scale": -INF}, {"scale": NAN}, {"scale": 3e38}], ids=str)
def test_prompt_refuses(nt, kw):   # noqa: F811
    assert prompt(nt, **kw) == nt.NT_E_INVALID


def test_prompt_accepts_nothing_to_do_and_refuses_too_much(nt):   # noqa: F811
    assert prompt(nt) == nt.NT_OK
    assert prompt(nt, n_seqs=5) == nt.NT_OK and prompt(nt, n_rows=5) == nt.NT_OK
    assert prompt(nt, n_seqs=1, n_rows=2 ** 31 - 1) == nt.NT_E_UNSUPPORTED
    assert prompt(nt, n_seqs=2 ** 30 + 1, n_rows=1) == nt.NT_E_UNSUPPORTED
    assert prompt(nt, kv_ld=1 << 23) == nt.NT_OK and prompt(nt, dtype=0, kv_ld=1 << 22) == nt.NT_OK
    assert prompt(nt, kv_ld=(1 << 23) + 8) == nt.NT_E_UNSUPPORTED
    assert prompt(nt, dtype=0, kv_ld=(1 << 22) + 4) == nt.NT_E_UNSUPPORTED
    assert prompt(nt, n_seqs=1, n_rows=1 << 24, n_heads=65536, q_ld=65536 * 64, out_ld=65536 * 64) == nt.NT_E_UNSUPPORTED


@pytest.mark.parametrize("kw", [
    {"q": None}, {"lens": None}, {"out": None}, {"n_heads": 0}, {"n_heads": 3}, {"n_seqs": -1}, {"n_rows": -1},
    {"max_new": -1}, {"max_len": -1}, {"q_ld": 255}, {"out_ld": 248}, {"q_ld": 260}, {"q": P + 8}, {"out": P + 4},
    {"scale": INF}, {"scale": NAN}, {"off": None, "n_rows": 3, "n_seqs": 2}], ids=str)
def test_tree_refuses(nt, kw):   # noqa: F811
    assert tree(nt, **kw) == nt.NT_E_INVALID


def test_tree_refuses_more(nt):   # noqa: F811
    assert tree(nt) == nt.NT_OK
    assert tree(nt, cache=False) == nt.NT_E_INVALID
    for bad in ({"d_head": 48}, {"page_len": 24}, {"page_len": 512}, {"dtype": 7}, {"n_kv_heads": 0}, {"d_k": None},
                {"d_table": None}):
        c = _cache(nt)
        for k, v in bad.items():
            setattr(c, k, v)
        assert tree(nt, cache=c) == nt.NT_E_INVALID, bad
        assert keep(nt, cache=c) == nt.NT_E_INVALID, bad
    c = _cache(nt)
    c.fp8, c.dtype = 1, 2
    assert tree(nt, cache=c) == nt.NT_E_UNSUPPORTED and keep(nt, cache=c) == nt.NT_E_UNSUPPORTED
    assert tree(nt, max_new=65) == nt.NT_E_UNSUPPORTED
    assert tree(nt, max_new=65, mask=None) == nt.NT_OK
    assert tree(nt, n_seqs=1 << 22, n_rows=1 << 22) == nt.NT_E_UNSUPPORTED
    assert tree(nt, n_seqs=1, n_rows=1 << 24, max_new=1 << 24, mask=None) == nt.NT_E_UNSUPPORTED


def test_tree_workspace(nt):   # noqa: F811
    c = _cache(nt)
    c.max_pages = 1 << 20
    size = lambda *a: nt.nt_op_attn_tree_workspace(c, *a)   # noqa: E731
    assert size(4, 0, 0, 8, 64) == 0 and size(4, 3, 24, 8, 64) == 0       # one part each
    assert size(4, 2048, 2048 * 8, 8, 100000) == 0                       # tasks enough
    one = size(4, 1, 8, 8, 100000)
    assert one > 0 and one % 256 == 0
    assert size(4, 1, 64, 64, 100000) > one
    assert tree(nt, cache=c, n_seqs=1, n_rows=8, max_len=100000, ws_bytes=0) == nt.NT_E_WORKSPACE
    assert str(one) in nt.load_library().nt_last_error().decode()
    assert tree(nt, cache=c, n_seqs=1, n_rows=8, max_len=100000, ws=P, ws_bytes=one - 1) == nt.NT_E_WORKSPACE
    assert tree(nt, cache=c, n_seqs=1, n_rows=8, max_len=100000, ws=P + 64, ws_bytes=one) == nt.NT_E_INVALID
    lib = nt.load_library()
    assert lib.nt_op_attn_tree_workspace(ctypes.byref(c), 4, 1, 8, 8, 64, None) == nt.NT_E_INVALID
    b = ctypes.c_size_t()
    assert lib.nt_op_attn_tree_workspace(ctypes.byref(c), 3, 1, 8, 8, 64, ctypes.byref(b)) == nt.NT_E_INVALID
    assert lib.nt_op_attn_tree_workspace(None, 4, 1, 8, 8, 64, ctypes.byref(b)) == nt.NT_E_INVALID


@pytest.mark.parametrize("kw", [
    {"page_len": 8}, {"page_len": 48}, {"page_len": 512}, {"n_pages": 0}, {"max_pages": 0}, {"table": None}, {"lens": None},
    {"add": None}, {"ring": None}, {"state": None}, {"n_seqs": -1}, {"max_rows": -1}], ids=str)
def test_resize_refuses(nt, kw):   # noqa: F811
    assert resize(nt, **kw) == nt.NT_E_INVALID
    assert resize(nt, n_seqs=65537) == nt.NT_E_UNSUPPORTED


@pytest.mark.parametrize("kw", [{"off": None}, {"lens": None}, {"path": None}, {"n_path": None}, {"add": None},
                                {"n_seqs": -1}, {"max_path": -1}], ids=str)
def test_keep_refuses(nt, kw):   # noqa: F811
    assert keep(nt, **kw) == nt.NT_E_INVALID
    assert keep(nt, cache=False) == nt.NT_E_INVALID
    assert keep(nt) == nt.NT_OK
    assert keep(nt, n_seqs=2 ** 31 - 1) == nt.NT_E_UNSUPPORTED


def test_the_statuses_are_the_headers(nt):   # noqa: F811
    import os
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "nt.h")).read()
    for name in ("NT_RESIZE_TABLE", "NT_RESIZE_ROWS"):
        assert int(re.search(r"#define %s \((-\d+)\)" % name, src).group(1)) == getattr(nt, name)
