"""Host-only checks of nt_op_token_logp: what it refuses, and its workspace sizes."""
import ctypes

import pytest

from tests.test_paged_cpu import P, nt   # noqa: F401  (the fixture)


def _call(nt, **kw):   # noqa: F811
    a = dict(dtype=0, x=P, ld=100, rows=2000, V=100, tokens=P, n_tok=1, k=4, logp=P, lse=P, ent=P, topi=P, toplp=P, ws=None, size=0)
    a.update(kw)
    return nt.load_library().nt_op_token_logp(a["dtype"], a["x"], a["ld"], a["rows"], a["V"], a["tokens"], a["n_tok"], a["k"],
                                              a["logp"], a["lse"], a["ent"], a["topi"], a["toplp"], a["ws"], a["size"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(x=None), 1), (dict(tokens=None), 1), (dict(logp=None), 1),
    (dict(topi=None), 1), (dict(toplp=None), 1), (dict(rows=-1), 1), (dict(V=0), 1), (dict(V=-5), 1), (dict(ld=99), 1),
    (dict(n_tok=-1), 1), (dict(x=P + 2), 1), (dict(dtype=1, x=P + 1), 1), (dict(k=-1), 2), (dict(k=33), 2),
    (dict(V=3, k=4), 2), (dict(rows=1 << 24), 2), (dict(rows=1, V=(1 << 30) + 1, ld=(1 << 30) + 1), 2),
    (dict(rows=1, V=100000, ld=100000), 3), (dict(rows=1, V=100000, ld=100000, ws=P, size=64), 3),
    (dict(rows=1, V=100000, ld=100000, ws=P + 16, size=1 << 20), 1),
    (dict(rows=0), 0), (dict(rows=0, n_tok=0, tokens=None, logp=None, k=0, topi=None, toplp=None, lse=None, ent=None), 0)])
def test_refusals(nt, kw, code):   # noqa: F811
    assert _call(nt, **kw) == code
    assert bool(nt.load_library().nt_last_error()) == (code != 0)


def test_workspace_sizes(nt):   # noqa: F811
    size = nt.nt_op_token_logp_workspace
    assert size("f32", 5000, 32000, 8) == 0 and size("f32", 1, 1000, 8) == 0 and size("f32", 1, 32000, 8) == 0 and size("bf16", 0, 100000, 8) == 0
    assert 0 < size("f32", 1, 1 << 30, 32) <= 32 * (4 + 64) * 4 + 256
    assert size("f32", 1, 100000, 32) % 256 == 0
    lib = nt.load_library()
    b = ctypes.c_size_t()
    assert lib.nt_op_token_logp_workspace(0, 1, 100, 4, None) == nt.NT_E_INVALID
    assert lib.nt_op_token_logp_workspace(9, 1, 100, 4, ctypes.byref(b)) == nt.NT_E_INVALID
    assert lib.nt_op_token_logp_workspace(0, 1, 100, 40, ctypes.byref(b)) == nt.NT_E_UNSUPPORTED
