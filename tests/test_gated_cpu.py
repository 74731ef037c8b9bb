"""Host-only checks of nt_op_gemm_gated: what it refuses, and which tiles it names."""
import pytest

from tests.test_paged_cpu import P, nt   # noqa: F401  (the fixture)


def _call(nt, **kw):   # noqa: F811
    a = dict(dtype=1, A=P, lda=128, Bt=P, M=0, N=64, K=128, act=0, bias=P, colsum=None, eps=1e-5, out=P, ldc=64)
    a.update(kw)
    return nt.load_library().nt_op_gemm_gated(a["dtype"], a["A"], a["lda"], a["Bt"], a["M"], a["N"], a["K"], a["act"],
                                              a["bias"], a["colsum"], a["eps"], a["out"], a["ldc"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(), 0), (dict(bias=None), 0), (dict(colsum=P), 0), (dict(eps=0.0), 0),
    (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(A=None), 1), (dict(Bt=None), 1), (dict(out=None), 1), (dict(M=-1), 1),
    (dict(N=0), 1), (dict(K=0), 1), (dict(K=96), 2), (dict(K=32, lda=32), 2), (dict(lda=127), 1), (dict(lda=132), 1),
    (dict(dtype=0, lda=130), 1), (dict(ldc=63), 1), (dict(A=P + 8), 1), (dict(Bt=P + 8), 1), (dict(out=P + 1), 1),
    (dict(act=4), 1), (dict(act=-1), 1), (dict(colsum=P, eps=0.0), 1), (dict(colsum=P, eps=-1.0), 1),
    (dict(colsum=P, eps=float("nan")), 1), (dict(N=1 << 24, ldc=1 << 24), 2), (dict(lda=1 << 24), 2)])
def test_refusals(nt, kw, code):   # noqa: F811
    assert _call(nt, **kw) == code
    assert bool(nt.load_library().nt_last_error()) == (code != 0)


def test_tiles(nt):   # noqa: F811
    rows = nt.nt_op_gemm_gated_rows
    assert rows("f16", 1, 64, 96) == rows("f16", -1, 64, 128) == rows("f16", 1, 0, 128) == -1
    assert rows("f16", 8, 1 << 24, 128) == -1
    # as many rows a launch as its offsets and its grid take
    assert rows("f16", 2 ** 31 - 1, 64, 64) == rows("f16", 1 << 24, 64, 64) == 256
    assert rows("f32", 2 ** 31 - 1, 1 << 20, 64) == 64
    seen = {(dt, ln): {rows(dt, m, 1024, 512, ln) for m in (1, 100, 500, 1024, 2300, 5000, 16384)}
            for dt in ("f16", "bf16", "f32") for ln in (False, True)}
    for dt in ("f16", "bf16"):
        assert seen[dt, False] == {32, 64, 128, 256} and seen[dt, True] == {32, 64, 128}
    assert seen["f32", False] == seen["f32", True] == {32, 64}
