"""GPU: nt_op_token_logp (log-probabilities of given tokens, log-sum-exp, entropy, best
alternatives) against float64.

Bounds, with n = V / 256 values a thread adds up: a sum of exponentials is off by at most
E = (n + 64) 2^-24 (its additions, those of the lanes and parts among them) + 2^-21 (the
exponential's own error and its rounded argument, |d| e^d 2^-24 with |d| e^d < 0.4, on both
sides), relative; its logarithm by E, plus two roundings of the results' sizes.  In the
entropy log s - t / s both sums are off by E relative, and -t / s is at most the entropy plus
log s, so at most 2 log V."""
import numpy as np
import pytest

from tests.paged_util import torch_dtype

pytestmark = pytest.mark.gpu
INT_MAX = np.iinfo(np.int32).max


def _run(x, tokens, k, V=None, want=("lse", "entropy"), ws=None, out=None):
    """x: [rows, V] torch tensor on the GPU (rows may be strided)."""
    import torch
    from paper_2109_08008_amd import nt
    name = {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}[x.dtype]
    rows, V = x.shape[0], V or x.shape[1]
    n_tok = tokens.shape[1]
    o = out or {"logp": torch.full((rows, n_tok), 77.0, device="cuda"), "lse": torch.full((rows,), 77.0, device="cuda"),
                "entropy": torch.full((rows,), 77.0, device="cuda"),
                "topi": torch.full((rows, k), -7, dtype=torch.int32, device="cuda"),
                "toplp": torch.full((rows, k), 77.0, device="cuda")}
    need = nt.nt_op_token_logp_workspace(name, rows, V, k)
    if ws is None:
        ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda")
    ptr = lambda t: t.data_ptr() if t.numel() else None   # noqa: E731
    nt.nt_op_token_logp(name, x.data_ptr(), x.stride(0), rows, V, ptr(tokens), n_tok, k, ptr(o["logp"]),
                        ptr(o["lse"]) if "lse" in want else None, ptr(o["entropy"]) if "entropy" in want else None,
                        ptr(o["topi"]), ptr(o["toplp"]), ws.data_ptr() if need else None, need)
    return o


def _expected(x, tokens, k):
    """float64, from the definition.  x: float64 numpy [rows, V]."""
    rows, V = x.shape
    m = x.max(1, keepdims=True)
    with np.errstate(all="ignore"):
        d = np.where(m == -np.inf, -np.inf, x - m)
        e = np.exp(d)
        s = e.sum(1, keepdims=True)
        lse = (m + np.log(s))[:, 0]
        ent = np.where(s[:, 0] == 0, 0.0, np.log(s[:, 0]) - np.where(e > 0, e * d, 0.0).sum(1) / s[:, 0])
        lp = np.where(x == -np.inf, -np.inf, d - np.log(s))     # (x - lse would lose log s beside 3e38)
    logp = np.zeros(tokens.shape)
    ok = (tokens >= 0) & (tokens < V)
    r, c = np.nonzero(ok)
    logp[r, c] = lp[r, tokens[r, c]]
    topi = np.full((rows, k), INT_MAX, dtype=np.int64)
    toplp = np.full((rows, k), -np.inf)
    for i in range(rows):
        best = np.lexsort((np.arange(V), -x[i]))[:k]
        best = best[x[i, best] > -np.inf]
        topi[i, :len(best)] = best
        toplp[i, :len(best)] = lp[i, best]
    return {"logp": logp, "lse": lse, "entropy": ent, "topi": topi, "toplp": toplp}


def _check(got, want, V, what=""):
    E = (V / 256 + 64) * 2.0 ** -24 + 2.0 ** -21
    np.testing.assert_array_equal(got["topi"].cpu().numpy(), want["topi"], err_msg=str(what))
    for name in ("logp", "lse", "entropy", "toplp"):
        g, w = got[name].cpu().numpy().astype(np.float64), want[name]
        fin = np.isfinite(w)
        np.testing.assert_array_equal(g[~fin], w[~fin], err_msg="%s %s" % (name, what))
        assert np.isfinite(g[fin]).all(), (name, what)
        big = np.abs(want["lse"])[np.isfinite(want["lse"])].max(initial=0.0) if name == "lse" else 0.0
        tol = E + 2.0 ** -22 * (1 + np.abs(w[fin]) + big)
        if name == "entropy":
            tol = E * (2 + 4 * np.log(V + 1)) + 2.0 ** -22 * (1 + np.log(V + 1))
        over = np.abs(g[fin] - w[fin]) - tol
        assert over.size == 0 or over.max() <= 0, (name, what, over.max())


def _logits(rows, V, kind, seed):
    rng = np.random.default_rng(seed)
    if kind == "normal":
        x = rng.standard_normal((rows, V)) * 4
    elif kind == "ties":
        x = rng.integers(0, 4, (rows, V)).astype(float)
    elif kind == "peaked":
        x = rng.standard_normal((rows, V)) - 30
        x[np.arange(rows), rng.integers(0, V, rows)] = 10.0
    elif kind == "masked":
        x = rng.standard_normal((rows, V)) * 3
        x[rng.random((rows, V)) < 0.7] = -np.inf
        x[0] = -np.inf
        if rows > 1:
            x[1] = -np.inf
            x[1, V // 2] = -3.0
        if rows > 2:
            x[2, : V // 2] = -np.inf
    elif kind == "offset":     # far from zero: x log2(e) is rounded by more than the probabilities may be
        x = rng.standard_normal((rows, V)) * 3 + np.where(np.arange(rows) % 2, -1.0, 1.0)[:, None] * 50000.0
    elif kind == "lowest":     # ruled out by the type's lowest value: the first half of the row at least
        x = rng.standard_normal((rows, V)) * 3
        x[:, : V // 2 + 1] = -np.inf       # (made finite by _case)
        x[rng.random((rows, V)) < 0.3] = -np.inf
        x[0] = -np.inf
    elif kind == "steps":      # one thread's values in 16 hold everything that is large, all different
        x = rng.standard_normal((rows, V)) - 20
        big = (np.arange(V) // 8) % 64 < 4
        x[:, big] = rng.permutation(np.linspace(1, 8, big.sum()))
    elif kind == "sorted":
        x = np.broadcast_to(np.linspace(6, -6, V), (rows, V)).copy()
        x[rows // 2:] = x[rows // 2:, ::-1]
    else:                      # constant rows, the last value best, the lowest of the type
        x = np.full((rows, V), 1.5)
        x[rows // 2:, -1] = 2.0
        x[-1] = -60000.0
    return x


def _case(rows, V, kind, dtype, k, n_tok, seed, pad=0):
    import torch
    x = torch.full((rows, V + pad), float("nan"), dtype=torch_dtype(dtype))
    x[:, :V] = torch.from_numpy(_logits(rows, V, kind, seed)).to(x.dtype)
    if kind == "lowest":
        x[:, :V] = x[:, :V].clamp(min=torch.finfo(x.dtype).min)
    rng = np.random.default_rng(seed + 1)
    tokens = rng.integers(0, V, (rows, n_tok)).astype(np.int32)
    if n_tok > 1:
        tokens[:, 0] = rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31], rows)
    x64 = x[:, :V].to(torch.float64).numpy()
    return x.cuda()[:, :V], torch.from_numpy(tokens).cuda(), _expected(x64, tokens, k)


KINDS = ["normal", "ties", "peaked", "masked", "steps", "sorted", "constant", "lowest", "offset"]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,V,k,n_tok", [(3, 1, 1, 1), (5, 7, 7, 2), (4, 33, 5, 0), (9, 101, 32, 3), (600, 255, 4, 1),
                                            (7, 1000, 8, 2), (5, 1021, 0, 1), (9, 1000, 32, 70), (6, 2048, 32, 1),
                                            (530, 2051, 20, 1), (9, 4099, 32, 1), (3, 8195, 32, 2),
                                            (6, 32000, 8, 300), (2, 65537, 20, 1), (1, 150001, 32, 1)])
def test_against_float64(rows, V, k, n_tok, kind, dtype):
    """Every length of head and tail (odd V: rows start at any alignment), rows shorter than a
    vector, cut and uncut, ties past what the collection holds, ruled-out words, constant rows,
    tokens outside the vocabulary, more tokens than threads."""
    x, tokens, want = _case(rows, V, kind, dtype, k, n_tok, V + rows, pad=(rows * 3) % 5)
    _check(_run(x, tokens, k), want, V, (kind, dtype))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,V,k", [(3, 190003, 22), (3, 190007, 23), (2, 200031, 32), (70, 180001, 1)])
def test_cut_rows(rows, V, k, kind, dtype):
    """Rows in parts on both sides of the alternatives that a merge takes as they are."""
    from paper_2109_08008_amd import nt
    assert nt.nt_op_token_logp_workspace(dtype, rows, V, k) > 0
    x, tokens, want = _case(rows, V, kind, dtype, k, 1, V + rows, pad=3)
    _check(_run(x, tokens, k), want, V, (kind, dtype))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,V,k", [(515, 2201, 20), (520, 2049, 32), (4100, 2153, 3)])
def test_many_rows_of_a_few_thousand(rows, V, k, kind, dtype):
    x, tokens, want = _case(rows, V, kind, dtype, k, 1, V + rows, pad=1)
    _check(_run(x, tokens, k), want, V, (kind, dtype))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,V,k", [(5, 12001, 32), (3, 16384, 1), (2, 33007, 20), (257, 12001, 5)])
def test_few_rows_of_many_values(rows, V, k, kind, dtype):
    x, tokens, want = _case(rows, V, kind, dtype, k, 2, V + rows, pad=1)
    _check(_run(x, tokens, k), want, V, (kind, dtype))


def test_cut_and_uncut_agree_on_alternatives():
    """The same rows alone (cut into parts) and among many (not cut)."""
    import torch
    from paper_2109_08008_amd import nt
    assert nt.nt_op_token_logp_workspace("f32", 1, 70000, 8) > 0 == nt.nt_op_token_logp_workspace("f32", 1100, 70000, 8)
    x, tokens, want = _case(1100, 70000, "normal", "f32", 8, 1, 5)
    many = _run(x, tokens, 8)
    for r in (0, 777, 1099):
        one = _run(x[r:r + 1], tokens[r:r + 1], 8)
        assert torch.equal(one["topi"][0], many["topi"][r])
        _check(one, {n: v[r:r + 1] for n, v in want.items()}, 70000)


@pytest.mark.parametrize("rows", [4, 2000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_and_nan(rows, dtype):
    """A NaN or +inf makes its own row's results NaN and nobody else's; a NaN is never chosen."""
    import torch
    V, k = 45000, 6
    x, tokens, want = _case(rows, V, "normal", dtype, k, 1, 3)
    x = x.clone()
    x[1, 12345] = float("nan")
    x[2, 44999] = float("inf")
    got = _run(x, tokens, k)
    for r in (1, 2):
        assert torch.isnan(got["lse"][r]) and torch.isnan(got["entropy"][r]) and torch.isnan(got["logp"][r]).all()
        assert torch.isnan(got["toplp"][r]).all()
    assert 12345 not in got["topi"][1].tolist() and got["topi"][2, 0] == 44999
    rest = [r for r in range(rows) if r not in (1, 2)]
    _check({n: v[rest] for n, v in got.items()}, {n: v[rest] for n, v in want.items()}, V)
    x[3] = float("nan")
    got = _run(x, tokens, k)
    assert torch.isnan(got["lse"][3]) and (got["topi"][3] == INT_MAX).all()


def test_outputs_that_are_not_asked_for():
    import torch
    x, tokens, want = _case(5, 3000, "normal", "f32", 4, 1, 1)
    for r in (5, 1):
        got = _run(x[:r], tokens[:r], 4, want=())
        assert (got["lse"] == 77).all() and (got["entropy"] == 77).all()
        np.testing.assert_array_equal(got["topi"].cpu().numpy(), want["topi"][:r])
        got = _run(x[:r], tokens[:r, :0], 0)
        np.testing.assert_allclose(got["lse"].cpu().numpy(), want["lse"][:r], rtol=1e-6)


def test_past_32_bit_offsets():
    """Rows beyond 2^32 elements."""
    import torch
    V, rows = 65536, (1 << 16) + 3
    x = torch.empty(rows, V, dtype=torch.bfloat16, device="cuda")
    x.fill_(-1.0)
    last = _logits(1, V, "normal", 1)
    x[-1] = torch.from_numpy(last[0]).to(torch.bfloat16)
    tokens = torch.full((rows, 1), 4321, dtype=torch.int32, device="cuda")
    got = _run(x, tokens, 3)
    w = _expected(x[-1:].cpu().to(torch.float64).numpy(), np.array([[4321]], dtype=np.int32), 3)
    _check({n: v[-1:] for n, v in got.items()}, w, V)
    assert (got["topi"][:-1].cpu() == torch.arange(3, dtype=torch.int32)).all()


@pytest.mark.parametrize("rows", [1, 40])
def test_captured_and_replayed(rows):
    import torch
    V, k = 100001, 8
    x, tokens, _ = _case(rows, V, "normal", "f16", k, 1, 2)
    x = x.contiguous()
    from paper_2109_08008_amd import nt
    ws = torch.empty(max(256, nt.nt_op_token_logp_workspace("f16", rows, V, k)), dtype=torch.uint8, device="cuda")
    out = _run(x, tokens, k, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        _run(x, tokens, k, ws=ws, out=out)
    for seed in range(3):
        x.copy_(torch.from_numpy(_logits(rows, V, KINDS[seed], seed)).half())
        graph.replay()
        eager = _run(x, tokens, k)
        torch.cuda.synchronize()
        assert all(torch.equal(out[n].view(torch.int32), eager[n].view(torch.int32)) for n in out)


def test_forced_decoding_is_scored():
    """The logits that nt_decode_step copies out of forced steps: the given tokens' log-probs are
    those that the decoder reports."""
    import synth
    import torch
    from paper_2109_08008_amd import nt
    from tests.gpu_util import gpu_encode, new_model
    w = synth.WORKLOADS["tiny"]
    ids, offs = synth.make_sentences(w.data, w.model.vocab, n_sent=5)
    src, V = synth.sentence_list(ids, offs), w.model.vocab
    model = new_model(w.model, synth.make_weights(w.model, lively=True), "f32")
    B, steps = len(src), 6
    search = synth.SearchSetup(beam=1, max_len_a=0.0, max_len_b=steps + 1, token_budget=0, prune=1)
    st, keep = gpu_encode(model, src, search)
    forced = torch.from_numpy(np.random.default_rng(1).integers(4, V, (steps, B)).astype(np.int32)).cuda()
    logits = torch.empty(B, V, device="cuda")
    scored = []
    for t in range(steps):
        nt.nt_decode_step(st, forced[t].data_ptr(), logits.data_ptr())
        got = _run(logits, forced[t].view(B, 1), 5)
        want = _expected(logits.cpu().to(torch.float64).numpy(), forced[t].view(B, 1).cpu().numpy(), 5)
        _check(got, want, V)
        scored.append(got["logp"][:, 0].cpu().numpy())
    nt.nt_decode_step(st, torch.full((B,), 2, dtype=torch.int32, device="cuda").data_ptr(), logits.data_ptr())
    toks, _, logp = nt.nt_dec_state_read(st)
    nt.nt_free_state(st)
    for b in range(B):
        np.testing.assert_array_equal(toks[b], forced[:, b].cpu().numpy())
        # two log-sum-exps of the same fp32 logits, each off by at most _check's bound
        np.testing.assert_allclose(logp[b], [s[b] for s in scored], rtol=2.0 ** -20, atol=2.0 ** -17)
    model.close()


def _far_from_zero(V, seed):
    """Rows whose largest values are far from zero: constant ones, among them those where the rounding
    error of x log2(e) is near -127 and near 127, and rows of neighbouring fp32 values below and above
    a base."""
    rng = np.random.default_rng(seed)
    base = [2041724160.0, 2727315712.0, -2041724160.0]
    base += (2.0 ** rng.uniform(20, 36, 20)).tolist() + (-2.0 ** rng.uniform(20, 36, 6)).tolist() + [3e37, -3e38]
    # the largest errors among some thousands of values
    many = np.float32(2.0 ** rng.uniform(30, 33, 20000)).astype(np.float32)
    r = many.astype(np.float64) * np.float64(np.float32(1.4426950408889634))
    r = r - r.astype(np.float32)
    base += many[np.argsort(r)[[0, 1, -2, -1]]].tolist() + many[np.argsort(np.abs(r - 64))[:2]].tolist()
    base = np.asarray(base, dtype=np.float32)
    x = np.repeat(base[:, None], V, 1)
    spread = rng.integers(-6, 1, x.shape) * np.spacing(np.abs(x))
    spread[:, rng.random(V) < 0.5] = 0.0
    x = np.concatenate([x, (x + spread).astype(np.float32)])
    x[1::5, rng.random(V) < 0.01] = -np.inf
    return x


@pytest.mark.parametrize("rows,V,k", [(74, 32000, 8), (74, 2000, 5), (4, 150016, 3), (700, 2304, 8), (4100, 2304, 0),
                                      (300, 12032, 20), (74, 12032, 0)])
def test_logits_far_from_zero(rows, V, k):
    """fp32 rows past 2^20 in size: one wave, two, four and sixteen waves a row, and cut; rows that start
    on 128-byte lines (every value in vectors)."""
    import torch
    x = _far_from_zero(V, V)
    x = np.resize(x, (rows, V)) if rows >= len(x) else x[[0, 1, 37, 38]]
    tokens = np.random.default_rng(1).integers(0, V, (rows, 2)).astype(np.int32)
    want = _expected(x.astype(np.float64), tokens, k)
    got = _run(torch.from_numpy(np.ascontiguousarray(x)).cuda(), torch.from_numpy(tokens).cuda(), k)
    # the log-sum-exp is the maximum and a logarithm, rounded once; everything else is of differences
    lse = got.pop("lse").cpu().numpy().astype(np.float64)
    E = (V / 256 + 64) * 2.0 ** -24 + 2.0 ** -21
    assert (np.abs(lse - want["lse"]) <= 2.0 ** -24 * np.abs(want["lse"]) + E + 2.0 ** -20).all()
    _check(got | {"lse": torch.from_numpy(want["lse"])}, want, V)
