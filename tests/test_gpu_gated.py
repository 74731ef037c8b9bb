"""GPU: nt_op_gemm_gated (both projections of a gated feed-forward block, activation and product in
one kernel, with or without the pre-norm LayerNorm folded in) against float64.

Bounds per element: with S = sum |a||b| (and the bias), a product of K terms summed in fp32 is off
by at most (K + 2) 2^-24 S; the activation's slope is at most 1.13, its own error 2^-19 of its
value (hardware exponential and reciprocal, or a few ulp of the library's); the result is rounded by
half a step of dtype.  A folded LayerNorm takes the row's statistics from fp32 sums of K terms: the
mean is off by dmu = (K + 2) 2^-24 times the values' mean size and two roundings; the variance is
the mean square less the mean's, off by (K + 8) 2^-24 (var + mean^2) + 2 |mean| dmu, and 1/std by
half that over var, relative.  Where mean^2 is more than about 64 var the kernel takes the
deviations from the mean instead: off by (K + 8) 2^-24 var + dmu^2."""
import numpy as np
import pytest

from tests.paged_util import EPS, torch_dtype

pytestmark = pytest.mark.gpu
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


def _act(g, name):
    import torch
    if name == "relu":
        return torch.relu(g)
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return g * 0.5 * (1 + torch.erf(g / 2 ** 0.5))
    return g * 0.5 * (1 + torch.tanh((2 / np.pi) ** 0.5 * (g + 0.044715 * g ** 3)))


def _inputs(dtype, M, N, K, ln, bias, seed, pad=0, outlier=0.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    a = torch.randn(M, K + pad, generator=g) * (1.5 if ln else 1.0) + (0.3 if ln else 0.0)
    if outlier:
        a[:, 0] = outlier
    w = torch.randn(2 * N, K, generator=g) * K ** -0.5
    a, w = a.to(torch_dtype(dtype)).cuda(), w.to(torch_dtype(dtype)).cuda()
    b = (torch.randn(2 * N, generator=g) * 0.5).cuda() if bias else None
    cs = w.double().sum(1).float() if ln else None
    return a[:, :K], w, b, cs


def _run(dtype, a, w, b, cs, act, out=None, eps=1e-5, ldc=None):
    import torch
    from paper_2109_08008_amd import nt
    M, K = a.shape
    N = w.shape[0] // 2
    if out is None:
        out = torch.full((M, ldc or N), 7.0, dtype=a.dtype, device="cuda")
    nt.nt_op_gemm_gated(dtype, a.data_ptr(), a.stride(0), w.data_ptr(), M, N, K, act, b.data_ptr() if b is not None else None,
                        out.data_ptr(), out.stride(0), d_colsum=cs.data_ptr() if cs is not None else None, ln_eps=eps)
    return out


def _expected(dtype, a, w, b, cs, act, eps=1e-5):
    import torch
    a, w = a.double(), w.double()
    M, K = a.shape
    N = w.shape[0] // 2
    u24 = 2.0 ** -24
    y, S = a @ w.t().contiguous(), a.abs() @ w.abs().t().contiguous()
    d = (K + 2) * u24 * S
    if cs is not None:
        cs = cs.double()
        mu = a.mean(1, keepdim=True)
        var = ((a - mu) ** 2).mean(1, keepdim=True)
        rs = 1 / torch.sqrt(var + eps)
        dmu = (K + 2) * u24 * a.abs().mean(1, keepdim=True) + 2 * u24 * mu.abs()
        r2 = mu ** 2 * rs ** 2
        by_squares = (K + 8) * u24 * (1 + r2) + mu.abs() * dmu * rs ** 2
        drs = torch.where(r2 > 70, (K + 8) * u24 + dmu ** 2 * rs ** 2, by_squares)
        y = rs * (y - mu * cs)
        d = rs * (d + dmu * cs.abs() + 4 * u24 * (mu * cs).abs()) + y.abs() * drs
    if b is not None:
        y = y + b.double()
    d = d + 4 * u24 * y.abs()
    g, u, dg, du = y[:, :N], y[:, N:], d[:, :N], d[:, N:]
    f = _act(g, act)
    out = f * u
    df = 1.13 * dg + 2.0 ** -19 * f.abs() + 2.0 ** -30
    bound = df * u.abs() + du * f.abs() + df * du + EPS[dtype] / 2 * out.abs() * (1 + 2.0 ** -10)
    if dtype == "f16":
        bound = bound + 2.0 ** -25
    return out, bound


def _check(dtype, got, a, w, b, cs, act, what=""):
    import torch
    want, bound = _expected(dtype, a, w, b, cs, act)
    got = got[:, :want.shape[1]].double()
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - bound
    assert float(over.max()) <= 0, (what, float(over.max()), float((got - want).abs().max()))


SHAPES = [(1, 16, 64), (1, 1, 128), (3, 5, 64), (17, 33, 192), (64, 100, 320), (65, 130, 128), (130, 1000, 576),
          (200, 2048, 512), (333, 999, 448), (700, 1024, 256), (2000, 1365, 512), (1111, 2730, 1024), (4100, 1408, 384)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("ln,bias", [(False, False), (False, True), (True, True), (True, False)])
def test_against_float64(dtype, M, N, K, ln, bias):
    """One token to thousands, N of every alignment, odd and even numbers of k-steps, every tile."""
    act = ACTS[(M + N + ln) % 4]
    a, w, b, cs = _inputs(dtype, M, N, K, ln, bias, M + N)
    _check(dtype, _run(dtype, a, w, b, cs, act), a, w, b, cs, act)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_activations_over_their_range(dtype, act):
    """Gates from the far negative to the far positive, up values of 1: the activation itself."""
    import torch
    N, K = 2048, 64
    a = torch.zeros(2, K, dtype=torch_dtype(dtype), device="cuda")
    a[:, 0], a[1, 0] = 1.0, -1.0
    w = torch.zeros(2 * N, K, dtype=a.dtype, device="cuda")
    w[:N, 0] = torch.linspace(-30, 30, N).to(a.dtype).cuda()
    b = torch.zeros(2 * N, device="cuda")
    b[N:] = 1.0
    _check(dtype, _run(dtype, a, w, b, None, act), a, w, b, None, act)
    # far beyond any exponential's range: act(g) is g or 0
    w[:N, 0] = torch.linspace(-60000, 60000, N).to(a.dtype).cuda()
    got = _run(dtype, a, w, b, None, act).float()
    want = torch.relu(torch.stack([w[:N, 0], -w[:N, 0]]).float())
    assert torch.equal(got[want > 100], want[want > 100]) and (got[want == 0].abs() <= 2.0 ** -20).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_infinities_and_nan_stay_in_their_rows(dtype):
    import torch
    a, w, b, cs = _inputs(dtype, 300, 256, 128, False, True, 3)
    a = a.contiguous()
    clean = _run(dtype, a, w, b, None, "silu")
    a[7, 5] = float("nan")
    a[150, 100] = float("inf")
    got = _run(dtype, a, w, b, None, "silu")
    rest = [r for r in range(300) if r not in (7, 150)]
    assert torch.equal(got[rest], clean[rest]) and torch.isnan(got[7]).all() and not torch.isfinite(got[150]).any()
    assert torch.isnan(_run(dtype, a, w, b, None, "relu")[7]).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_layernorm_of_awkward_rows(dtype):
    """A large first value (the statistics' shift), a large common offset, nearly constant rows."""
    import torch
    for seed, kw in ((1, dict(outlier=60.0)), (2, dict(outlier=-0.5))):
        a, w, b, cs = _inputs(dtype, 70, 96, 512, True, True, seed, **kw)
        a = a.contiguous()
        if seed == 2:
            a += 20.0
            a[3] = 2.0
            a[4] = 0.0
        _check(dtype, _run(dtype, a, w, b, cs, "gelu"), a, w, b, cs, "gelu", kw)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("N", [256, 250, 77])
def test_strides_and_what_lies_beside(dtype, N):
    """Rows of A and out apart from each other; nothing outside the N columns and M rows changes."""
    import torch
    M, K = 90, 192
    a, w, b, cs = _inputs(dtype, M, N, K, True, True, 5, pad=8)
    for ldc in (N, N + 3, N + 16):
        big = torch.full((M + 40, ldc), 7.0, dtype=a.dtype, device="cuda")
        _run(dtype, a, w, b, cs, "silu", out=big)
        _check(dtype, big[:M], a, w, b, cs, "silu", ldc)
        assert (big[M:] == 7).all() and (big[:, N:] == 7).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("ln", [False, True])
@pytest.mark.parametrize("N,K", [(1024, 512), (1024, 448), (4096, 128)])
def test_every_tile_gives_the_same_bits(dtype, ln, N, K):
    """The first rows of ever larger products: other tiles, the same results."""
    import torch
    from paper_2109_08008_amd import nt
    M = 17000
    a, w, b, cs = _inputs(dtype, M, N, K, ln, True, 9)
    first, seen = None, set()
    for m in (5, 300, 700, 2300, 5000, M):
        seen.add(nt.nt_op_gemm_gated_rows(dtype, m, N, K, ln))
        got = _run(dtype, a[:m], w, b, cs, "gelu_tanh")
        if first is None:
            first = got
        assert torch.equal(got[:5], first), (m, seen)
    assert len(seen) >= 2


def test_past_32_bit_offsets():
    """A and out beyond 2^32 bytes: rows far apart, and as many as that."""
    import torch
    M, N, K, lda = 2500, 64, 128, 1 << 20
    buf = torch.empty(M * lda, dtype=torch.float16, device="cuda")
    a = buf.view(M, lda)[:, :K]
    src, w, b, _ = _inputs("f16", M, N, K, False, True, 2)
    a.copy_(src)
    _check("f16", _run("f16", a, w, b, None, "silu"), src, w, b, None, "silu")
    out = torch.empty(M, lda, dtype=torch.float16, device="cuda")
    _run("f16", src, w, b, None, "silu", out=out)
    _check("f16", out[:, :N], src, w, b, None, "silu")


@pytest.mark.parametrize("M", [2, 900])
def test_captured_and_replayed(M):
    import torch
    a, w, b, cs = _inputs("bf16", M, 512, 256, True, True, 4)
    a = a.contiguous()
    out = _run("bf16", a, w, b, cs, "silu")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        _run("bf16", a, w, b, cs, "silu", out=out)
    for seed in range(3):
        a.copy_(_inputs("bf16", M, 512, 256, True, True, 20 + seed)[0])
        graph.replay()
        want = _run("bf16", a, w, b, cs, "silu")
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("M,N,K", [(70, 96, 192), (300, 250, 448), (1100, 640, 960), (130, 1000, 1088)])
def test_fp32_layernorm_keeps_the_variance(M, N, K):
    """fp32 rows whose mean is 5 to 8 deviations from zero, of whole numbers, so that every sum is exact, and
    weights that pick one value each: what is left are the roundings of the mean and the variance.

    With u = 2^-24 and z the first value's distance from the mean in deviations: the mean less the
    first value is off by 2 u of itself, the mean square by 2 u, its square by 5 u: together
    u (3 + 7 z^2) of the variance, half of that in 1/std, whose root and quotient add 2 u; the mean is
    rounded by u mean + 2 u z std, the value less the mean once and the result twice."""
    import torch
    rng = np.random.default_rng(K)
    a = np.clip(72 + 10 * np.round(rng.standard_normal((M, K))), 32, 112)
    a[:, 0] = rng.choice([62.0, 72.0, 82.0], M)
    a = torch.from_numpy(a).float().cuda()
    pick = torch.from_numpy(rng.integers(0, K, N)).cuda()
    w = torch.zeros(2 * N, K, device="cuda")
    w[torch.arange(N, device="cuda"), pick] = 1.0
    b = torch.zeros(2 * N, device="cuda")
    b[N:] = 1.0
    cs = torch.cat([torch.ones(N), torch.zeros(N)]).cuda()
    got = _run("f32", a, w, b, cs, "relu").double()
    x = a.double()
    mu = x.mean(1, keepdim=True)
    rs = 1 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + 1e-5)
    want = torch.relu((x[:, pick] - mu) * rs)
    u, z2 = 2.0 ** -24, ((x[:, :1] - mu) * rs) ** 2
    assert float(z2.max()) < 4 and float((mu * rs).min()) > 5
    tol = u * (mu * rs + 2 * z2.sqrt()) + want * u * (1.5 + 3.5 * z2 + 2 + 3) + 2.0 ** -40
    over = (got - want).abs() - tol * (1 + 2.0 ** -10)
    assert float(over.max()) <= 0, (float(over.max() / u), float((got - want).abs().max() / u))


def _awkward(dtype, M, N, K, seed):
    """Rows of every kind that the statistics tell apart, side by side: ordinary ones, a common offset of
    13 deviations in every third, of 20 in whole blocks of 40, a far first value, constant ones."""
    import torch
    a, w, b, cs = _inputs(dtype, M, N, K, True, True, seed)
    a = a.contiguous()
    a[1::3] += 20.0
    a[100:140] += 30.0
    a[-45:-5] -= 30.0
    a[4::7, 0] = 60.0
    a[5] = 2.0
    a[M // 2] = 0.0
    return a, w, b, cs


@pytest.mark.parametrize("dtype,M,N,K,rows", [
    ("f32", 70, 96, 512, 32), ("f32", 1111, 2050, 320, 64),
    ("f16", 150, 96, 512, 32), ("f16", 1203, 2050, 576, 64), ("f16", 2165, 4100, 320, 128),
    ("bf16", 150, 96, 512, 32), ("bf16", 1203, 2050, 576, 64), ("bf16", 2165, 4100, 320, 128)])
def test_layernorm_of_awkward_rows_on_every_tile(dtype, M, N, K, rows):
    """Rows that are read a second time among ones that are not, on each tile that folds a LayerNorm in:
    every element against float64, and the first rows with the bits of the smallest tile."""
    import torch
    from paper_2109_08008_amd import nt
    assert nt.nt_op_gemm_gated_rows(dtype, M, N, K, True) == rows
    a, w, b, cs = _awkward(dtype, M, N, K, M)
    got = _run(dtype, a, w, b, cs, "gelu")
    _check(dtype, got, a, w, b, cs, "gelu")
    few = 20
    assert nt.nt_op_gemm_gated_rows(dtype, few, N, K, True) in (32, 64)
    assert torch.equal(got[:few], _run(dtype, a[:few], w, b, cs, "gelu"))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(2000, 4095, 576), (2000, 4001, 64), (2000, 4096, 128), (4000, 2000, 448),
                                   (3900, 2043, 192), (8000, 1021, 448)])
def test_the_largest_tile(dtype, M, N, K):
    """256x256 tiles with ragged rows and columns, one k-step, odd and even numbers of them: every
    element against float64, nothing beside the columns or behind the rows changed, and the first and
    last rows alone, on other tiles and at other places of one, with the same bits."""
    import torch
    from paper_2109_08008_amd import nt
    assert nt.nt_op_gemm_gated_rows(dtype, M, N, K) == 256
    act = ACTS[(M + N + K) % 4]
    a, w, b, _ = _inputs(dtype, M, N, K, False, N % 3 > 0, K)
    big = torch.full((M + 60, N + 3), 7.0, dtype=a.dtype, device="cuda")
    got = _run(dtype, a, w, b, None, act, out=big)[:M, :N]
    _check(dtype, got, a, w, b, None, act)
    assert (big[M:] == 7).all() and (big[:, N:] == 7).all()
    seen = set()
    for m in (20, 300, M // 2):
        seen.add(nt.nt_op_gemm_gated_rows(dtype, m, N, K))
        assert torch.equal(got[:m], _run(dtype, a[:m], w, b, None, act)), m
        assert torch.equal(got[-m:], _run(dtype, a[-m:], w, b, None, act)), m
    assert {32, 128} <= seen and 256 not in seen


@pytest.mark.parametrize("dtype,M,N,K", [("f32", 70, 96, 192), ("f32", 1100, 2050, 320), ("f16", 70, 96, 192), ("f16", 1203, 2050, 192),
                                         ("bf16", 70, 96, 192), ("bf16", 1203, 2050, 192), ("bf16", 2165, 4100, 192)])
def test_layernorm_of_rows_that_are_not_finite(dtype, M, N, K):
    """A row that holds a NaN or an infinity has no mean: all its results are NaN, and nobody else's.  Rows
    whose squares leave fp32 (or whose mean's does) have the variance inf, as two turns over them find it."""
    import torch
    a, w, b, cs = _inputs(dtype, M, N, K, True, True, M)
    a = a.contiguous()
    clean = _run(dtype, a, w, b, cs, "silu")
    bad = {3: float("nan"), 20: float("inf"), 41: -float("inf"), M - 1: float("inf")}
    for i, (r, x) in enumerate(bad.items()):
        a[r, (0, K // 2, 0, K - 1)[i]] = x
    huge = [] if dtype == "f16" else [10, 50]
    if huge:
        a[10] = a[10] * 1e25
        a[50] = a[50] * 1e22 + 1e25
    got = _run(dtype, a, w, b, cs, "silu")
    rest = [r for r in range(M) if r not in bad and r not in huge]
    assert torch.equal(got[rest], clean[rest])
    assert torch.isnan(got[list(bad)]).all()
    if huge:    # (x - mean) / inf = 0: the bias alone
        want = (torch.nn.functional.silu(b[:N].double()) * b[N:].double())[None]
        tol = EPS[dtype] / 2 * want.abs() * (1 + 2.0 ** -10) + 2.0 ** -18 * want.abs() + 2.0 ** -60
        assert ((got[huge].double() - want).abs() <= tol).all()
