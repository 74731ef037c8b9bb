"""Host-only checks of the paged cache's entry points: what they refuse, and with which status.
The addresses given are never touched."""
import ctypes
import os

import pytest

P = 1 << 20     # an aligned address


@pytest.fixture(scope="module")
def nt():
    from paper_2109_08008_amd import nt as _nt
    if not os.path.exists(_nt.LIB_PATH):
        from paper_2109_08008_amd.build import build_library
        build_library()
    _nt.load_library()
    return _nt


def _cache(nt, **kw):
    c = nt.kv_pages("f16", 2, 64, 16, 10, 4, P, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHE = [(dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(fp8=2), 1), (dict(fp8=1, dtype=0), 2), (dict(fp8=1, dtype=2), 2),
             (dict(d_head=16), 1), (dict(d_head=96), 1), (dict(d_head=256), 1), (dict(page_len=8), 1), (dict(page_len=48), 1),
             (dict(page_len=512), 1), (dict(page_len=0), 1), (dict(page_len=-16), 1), (dict(n_kv_heads=0), 1),
             (dict(n_kv_heads=5000), 1), (dict(n_pages=0), 1), (dict(max_pages=0), 1), (dict(max_pages=-2), 1)]
BAD_POOLS = [(dict(d_k=None), 1), (dict(d_v=None), 1), (dict(d_table=None), 1), (dict(d_k=P + 8), 1), (dict(d_v=P + 2), 1)]


def _append(nt, c, **kw):
    a = dict(d_k=P, d_v=P, ld=128, d_off=P, d_lens=P, n_seqs=3, n_rows=7)
    a.update(kw)
    return nt.load_library().nt_op_kv_append(ctypes.byref(c) if c else None, a["d_k"], a["d_v"], a["ld"], a["d_off"],
                                             a["d_lens"], a["n_seqs"], a["n_rows"], None)


def _attn(nt, c, **kw):
    a = dict(d_q=P, q_ld=256, n_heads=4, d_lens=P, n_seqs=3, max_len=64, scale=0.1, d_out=P, out_ld=256, d_ws=None,
             ws_bytes=0)
    a.update(kw)
    return nt.load_library().nt_op_attn_paged(ctypes.byref(c) if c else None, a["d_q"], a["q_ld"], a["n_heads"], a["d_lens"],
                                              a["n_seqs"], a["max_len"], a["scale"], a["d_out"], a["out_ld"], a["d_ws"],
                                              a["ws_bytes"], None)


@pytest.mark.parametrize("kw,code", BAD_CACHE + BAD_POOLS)
def test_caches_that_cannot_be(nt, kw, code):
    for call in (_append, _attn):
        assert call(nt, _cache(nt, **kw)) == code
        assert nt.load_library().nt_last_error()
    b = ctypes.c_size_t()
    got = nt.load_library().nt_op_attn_paged_workspace(ctypes.byref(_cache(nt, **kw)), 4, 3, 64, ctypes.byref(b))
    assert got == (code if (kw, code) in BAD_CACHE else 0)      # sizes need no pools


@pytest.mark.parametrize("kw", [dict(d_k=None), dict(d_v=None), dict(d_lens=None), dict(n_seqs=-1), dict(n_rows=-1),
                                dict(d_off=None), dict(ld=127), dict(ld=132), dict(d_k=P + 2), dict(d_v=P + 8)])
def test_append_refuses(nt, kw):
    assert _append(nt, _cache(nt), **kw) == nt.NT_E_INVALID


def test_append_sizes_past_its_indices(nt):
    for kw in (dict(n_rows=(1 << 30) + 1), dict(n_seqs=(1 << 30) + 1)):
        assert _append(nt, _cache(nt), **kw) == nt.NT_E_UNSUPPORTED


@pytest.mark.parametrize("kw,code", [
    (dict(d_q=None), 1), (dict(d_out=None), 1), (dict(d_lens=None), 1), (dict(n_seqs=-1), 1), (dict(max_len=-1), 1),
    (dict(n_heads=0), 1), (dict(n_heads=3), 1), (dict(n_heads=-2), 1), (dict(q_ld=255), 1), (dict(out_ld=248), 1),
    (dict(q_ld=260), 1), (dict(d_q=P + 4), 1), (dict(d_out=P + 4), 1), (dict(n_seqs=1 << 22), 2),
    (dict(n_seqs=1 << 30, n_heads=2, q_ld=128, out_ld=128), 2)])
def test_attention_refuses(nt, kw, code):
    assert _attn(nt, _cache(nt), **kw) == code


def test_null_caches_and_empty_calls(nt):
    assert _append(nt, None) == nt.NT_E_INVALID and _attn(nt, None) == nt.NT_E_INVALID
    lib = nt.load_library()
    assert lib.nt_op_attn_paged_workspace(ctypes.byref(_cache(nt)), 4, 3, 64, None) == nt.NT_E_INVALID
    assert _append(nt, _cache(nt), n_seqs=0, n_rows=0) == nt.NT_OK
    assert _append(nt, _cache(nt), n_rows=0) == nt.NT_OK
    assert _attn(nt, _cache(nt), n_seqs=0) == nt.NT_OK


def test_workspace_sizes(nt):
    """Nothing where a call is one launch; otherwise the parts' sums, and no more however far the
    lengths reach."""
    c = _cache(nt, max_pages=1 << 20, n_pages=1 << 20)
    size = lambda n, m: nt.nt_op_attn_paged_workspace(c, 4, n, m)   # noqa: E731
    assert size(0, 100) == 0 and size(5000, 250) == 0 and size(1, 0) == 0 and size(4, 100) == 0
    assert size(1, 100000) % 256 == 0 and size(1, 100000) > 0
    for n in (1, 7, 5000):      # a part of a task holds two heads' sums; 32768 parts and one a task at most
        assert size(n, 1 << 24) <= (32768 + 2 * n) * 2 * 66 * 4 + 256
    assert size(1, 2 ** 31 - 1) == size(1, 1 << 24)     # the table's reach
    wide = _cache(nt, max_pages=2 ** 31 - 1, page_len=256)
    assert nt.nt_op_attn_paged_workspace(wide, 2, 1 << 21, 2 ** 31 - 1) == 0   # one part each
    assert nt.nt_op_attn_paged_workspace(_cache(nt), 4, 1, 1 << 24) == 0     # 64 positions
    for bad in ((3, 1, 10), (4, -1, 10), (4, 1, -1)):
        with pytest.raises(nt.NTError):
            nt.nt_op_attn_paged_workspace(c, *bad)


def test_struct_matches_header(nt):
    import re
    from tests.test_abi_cpu import ROOT
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "nt.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\}\s*nt_kv_pages\s*;", src).group(1)
    names = []
    for decl in filter(None, (d.strip() for d in body.split(";"))):
        kind = "int32_t" if decl.startswith("int32_t") else "pointer"
        names += [(n.strip(" *"), kind) for n in decl.replace("const", "").split(None, 1)[1].split(",")]
    fields = nt.nt_kv_pages._fields_
    assert [n for n, _ in names] == [n for n, _ in fields]
    assert ["int32_t" if t is ctypes.c_int32 else "pointer" for _, t in fields] == [k for _, k in names]
