"""GPU: nt_op_attn_prompt, attention over packed sequences, against float64."""
import pytest

from tests.paged_util import torch_dtype
from tests.rows_util import assert_rows, attention

pytestmark = pytest.mark.gpu


def offsets(lens, first=0):
    off = [first]
    for n in lens:
        off.append(off[-1] + n)
    return off


def make(lens, heads, kv_heads, d_head, dtype, seed=0, first=0, behind=0, pad=0, scale=1.0):
    """Packed rows of query, key and value side by side; NaN in the rows of no sequence and between rows."""
    import torch
    g = torch.Generator().manual_seed(seed)
    off = offsets(lens, first)
    rows = off[-1] + behind
    width = (heads + 2 * kv_heads) * d_head
    x = torch.full((max(rows, 1), width + pad), float("nan"))
    x[first:off[-1], :width] = torch.randn(off[-1] - first, width, generator=g) * scale
    return x.to(torch_dtype(dtype)).cuda(), off, rows


def run(x, off, rows, heads, kv_heads, d_head, dtype, causal, scale, out=None, d_off=None, stream=None):
    import torch
    from paper_2109_08008_amd import nt
    eb = x.element_size()
    if out is None:
        out = torch.full((max(rows, 1), heads * d_head), 7.0, dtype=x.dtype, device=x.device)
    if d_off is None:
        d_off = torch.tensor(off, dtype=torch.int32, device=x.device)
    base = x.data_ptr()
    nt.nt_op_attn_prompt(dtype, base, x.stride(0), heads, base + heads * d_head * eb,
                         base + (heads + kv_heads) * d_head * eb, x.stride(0), kv_heads, d_head, d_off.data_ptr(),
                         len(off) - 1, rows, causal, scale, out.data_ptr(), out.stride(0), stream)
    return out


def split(x, heads, kv_heads, d_head):
    x = x.double()
    q = x[:, :heads * d_head].reshape(-1, heads, d_head)
    k = x[:, heads * d_head:(heads + kv_heads) * d_head].reshape(-1, kv_heads, d_head)
    v = x[:, (heads + kv_heads) * d_head:(heads + 2 * kv_heads) * d_head].reshape(-1, kv_heads, d_head)
    return q, k, v


def check(got, x, off, heads, kv_heads, d_head, dtype, causal, scale, what=""):
    import torch
    q, k, v = split(x, heads, kv_heads, d_head)
    for b in range(len(off) - 1):
        lo, hi = off[b], off[b + 1]
        if lo == hi:
            continue
        seen = torch.ones(hi - lo, hi - lo, dtype=torch.bool, device=x.device)
        if causal:
            seen = seen.tril()
        want, bound = attention(q[lo:hi], k[lo:hi], v[lo:hi], seen, scale, dtype)
        assert_rows(got[lo:hi].reshape(hi - lo, heads, d_head), want, bound, (what, b, hi - lo))
    untouched = torch.cat([got[:off[0]], got[off[-1]:]])
    assert bool((untouched == 7.0).all()), "rows of no sequence were written"


RAGGED = [0, 5, 0, 130, 64, 1, 1, 0, 63, 65]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("lens", [[1], [77], [16], [64], [129], RAGGED, [300, 17, 513], [3, 1000]], ids=str)
def test_lengths(lens, dtype, causal):
    h, hkv, dh = 4, 2, 64
    x, off, rows = make(lens, h, hkv, dh, dtype, seed=len(lens), behind=5)
    check(run(x, off, rows, h, hkv, dh, dtype, causal, dh ** -0.5), x, off, h, hkv, dh, dtype, causal, dh ** -0.5)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d_head", [32, 64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (6, 2), (20, 1)])
def test_heads(heads, kv_heads, d_head, dtype):
    x, off, rows = make([45, 200, 7], heads, kv_heads, d_head, dtype, seed=heads, first=2, behind=3, pad=16)
    scale = 1.3 * d_head ** -0.5
    check(run(x, off, rows, heads, kv_heads, d_head, dtype, True, scale), x, off, heads, kv_heads, d_head, dtype, True, scale)


@pytest.mark.parametrize("n_seqs,longest", [(64, 9), (65, 5), (700, 12), (5000, 2)])
def test_many_short_sequences(n_seqs, longest):
    lens = [(i * 7919) % (longest + 1) for i in range(n_seqs)]
    for causal in (True, False):
        x, off, rows = make(lens, 2, 1, 32, "f16", seed=n_seqs, behind=1)
        got = run(x, off, rows, 2, 1, 32, "f16", causal, 0.2)
        # one reference for all: row i sees key j of its own sequence only
        import torch
        seq = torch.repeat_interleave(torch.arange(n_seqs), torch.tensor(lens)).cuda()
        at = torch.arange(rows - 1, device="cuda")
        seen = seq[:, None] == seq[None, :]
        if causal:
            seen &= at[None, :] <= at[:, None]
        q, k, v = split(x[:rows - 1], 2, 1, 32)
        want, bound = attention(q, k, v, seen, 0.2, "f16")
        assert_rows(got[:rows - 1].reshape(-1, 2, 32), want, bound)
        assert bool((got[rows - 1:] == 7.0).all())


@pytest.mark.parametrize("n_seqs,every", [(4096, 63), (4097, 1000), (300000, 4099), (1 << 20, 99991)])
def test_few_tokens_in_many_sequences(n_seqs, every):
    """Most sequences are empty: a row's is found among many equal offsets."""
    import torch
    lens = torch.zeros(n_seqs, dtype=torch.int64)
    lens[every // 2::every] = torch.arange(len(lens[every // 2::every])) % 7 + 1
    lens[-1] = 5
    off = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)])
    short = [int(x) for x in lens[lens > 0]]
    x, packed, rows = make(short, 2, 1, 32, "f16", seed=n_seqs, behind=3)
    got = run(x, off.tolist(), rows, 2, 1, 32, "f16", True, 0.2)
    check(got, x, packed, 2, 1, 32, "f16", True, 0.2)


@pytest.mark.parametrize("lens", [[4000], [2048, 1, 3000]], ids=str)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_long(lens, dtype):
    x, off, rows = make(lens, 2, 1, 128, dtype, seed=9)
    check(run(x, off, rows, 2, 1, 128, dtype, True, 128 ** -0.5), x, off, 2, 1, 128, dtype, True, 128 ** -0.5)


TILES = [(96, 32, [1000, 1, 0, 23]), (64, 16, [300, 0, 129, 65, 6]), (40, 8, [150, 1, 31, 97, 41]), (12, 4, [77, 16, 33, 2]),
         (96, 32, [33, 1, 16, 0, 140, 64, 17, 63, 65, 2] * 3), (24, 8, [40, 1, 17, 33, 16, 15, 65, 2])]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("d_head", [32, 64, 128])
@pytest.mark.parametrize("heads,kv_heads,lens", TILES, ids=["128", "64", "32", "16", "short", "pair"])
def test_each_tile(heads, kv_heads, lens, d_head, dtype, causal):
    """Heads and rows enough for tiles of 128, 64, 32 and 16 rows and those of short sequences, which ends cut; behind the
    last sequence, and in its last token's value, stands no number."""
    import torch
    x, off, rows = make(lens, heads, kv_heads, d_head, dtype, seed=heads, behind=7)
    part = (heads + kv_heads) * d_head
    last = off[-1] - 1
    x[last, part:] = float("nan")
    scale = d_head ** -0.5
    got = run(x, off, rows, heads, kv_heads, d_head, dtype, causal, scale)
    lo = off[-2]                    # the last sequence's rows: all of them see it, or with causal the last alone
    hit = got[last if causal else lo:last + 1]
    assert bool(torch.isnan(hit).all())
    clean = x.clone()
    clean[last, part:] = 0
    q, k, v = split(clean, heads, kv_heads, d_head)
    for b in range(len(lens)):
        lo, hi = off[b], off[b + 1]
        if lo == hi:
            continue
        seen = torch.ones(hi - lo, hi - lo, dtype=torch.bool, device="cuda")
        want, bound = attention(q[lo:hi], k[lo:hi], v[lo:hi], seen.tril() if causal else seen, scale, dtype)
        n = hi - lo if b + 1 < len(lens) else (hi - lo - 1 if causal else 0)
        if n:
            assert_rows(got[lo:lo + n].reshape(n, heads, d_head), want[:n], bound[:n], (b, hi - lo))
    assert bool((got[off[-1]:] == 7.0).all())


@pytest.mark.parametrize("scale", [-0.125, 0.0, 4.0])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_scales(scale, dtype):
    x, off, rows = make([90, 150], 2, 2, 64, dtype, seed=3)
    check(run(x, off, rows, 2, 2, 64, dtype, True, scale), x, off, 2, 2, 64, dtype, True, scale)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("step", [0.02, 0.5, -0.5])
def test_scores_that_rise_and_fall(step, dtype):
    """The reference that scores are taken against moves late, often, or never again."""
    import torch
    n, dh = 500, 64
    x, off, rows = make([n], 1, 1, dh, dtype, seed=5, scale=0.1)
    x[:, :dh] = 0.0
    x[:, 0] = 1.0
    x[:, dh:2 * dh] = 0.0
    x[:, dh] = (torch.arange(n) * step).to(x.dtype).cuda()
    check(run(x, off, rows, 1, 1, dh, dtype, True, 1.0), x, off, 1, 1, dh, dtype, True, 1.0)


def test_a_long_tail_keeps_its_weight():
    """One key 14 above 4000 equal ones: they hold a third of one percent together."""
    n, dh = 4001, 64
    x, off, rows = make([n], 1, 1, dh, "f16", seed=6)
    x[:, :2 * dh] = 0.0
    x[:, 0] = 1.0
    x[0, dh] = 14.0
    x[:, 2 * dh:] = 0.0
    x[1:, 2 * dh:] = 1.0
    got = run(x, off, rows, 1, 1, dh, "f16", True, 1.0)
    check(got, x, off, 1, 1, dh, "f16", True, 1.0)
    assert 3e-3 < float(got[-1].float().mean()) < 4e-3


@pytest.mark.parametrize("dtype,size", [("f16", 1e4), ("bf16", 1e6), ("bf16", 1e15), ("f32", 1e6), ("f32", 1e15)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_past_two_to_the_31(sign, dtype, size):
    """A token that sees itself alone is its value (to the rounding of a division), however large its score."""
    import torch
    from tests.paged_util import EPS
    n, h, dh = 300, 4, 64
    x, off, rows = make([1] * n, h, h, dh, dtype, seed=12)
    x[:, :h * dh] *= size
    x[:, h * dh:2 * h * dh] *= size
    got = run(x, off, rows, h, h, dh, dtype, True, sign * 0.7).double()
    want = x[:, 2 * h * dh:].double()
    assert bool(((got - want).abs() <= (EPS[dtype] / 2 + 2.0 ** -22) * want.abs()).all())
    # and two of them, whose scores differ by a good part of themselves: the larger one's value
    x, off, rows = make([2] * n, 1, 1, dh, dtype, seed=13)
    x[:, :2 * dh] *= size
    x[1::2, dh:2 * dh] = x[0::2, dh:2 * dh] * -1
    got = run(x, off, rows, 1, 1, dh, dtype, False, sign * 0.7).double()
    q, k, v = split(x, 1, 1, dh)
    first = (q[:, 0] * k[::2, 0].repeat_interleave(2, 0)).sum(1) * sign > 0
    want = torch.where(first[:, None], v[::2, 0].repeat_interleave(2, 0), v[1::2, 0].repeat_interleave(2, 0))
    assert bool(((got - want).abs() <= (EPS[dtype] / 2 + 2.0 ** -22) * want.abs()).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("what", ["nan_value", "inf_value", "nan_key", "inf_key"])
def test_numbers_stay_with_the_rows_that_see_them(what, dtype):
    """A token whose key or value is no number: rows before it and other sequences do not notice."""
    import torch
    lens, h, hkv, dh = [40, 100, 30], 2, 1, 64
    x, off, rows = make(lens, h, hkv, dh, dtype, seed=8)
    bad = off[1] + 50
    part = (h + hkv) * dh if "value" in what else h * dh
    x[bad, part + 3] = float("nan") if "nan" in what else float("inf")
    got = run(x, off, rows, h, hkv, dh, dtype, True, 0.1)
    if "key" in what:       # the rows that see it are no numbers, or (a score of -inf) do not notice either
        q = x[bad:off[2], :h * dh].reshape(-1, h, dh)[:, :, 3].double()
        hit = torch.ones_like(q, dtype=torch.bool) if "nan" in what else q > 0
        seen_rows = got[bad:off[2]].reshape(-1, h, dh)
        assert bool(torch.isnan(seen_rows[hit]).all())
        clean = x.clone()
        clean[bad, part + 3] = 0
        qd, k, v = split(clean, h, hkv, dh)
        seen = torch.ones(100, 100, dtype=torch.bool, device="cuda").tril()
        want, bound = attention(qd[off[1]:off[2]], k[off[1]:off[2]], v[off[1]:off[2]], seen, 0.1, dtype)
        assert_rows(got[off[1]:bad].reshape(-1, h, dh), want[:50], bound[:50], what)
        seen[:, 50] = False
        want, bound = attention(qd[off[1]:off[2]], k[off[1]:off[2]], v[off[1]:off[2]], seen, 0.1, dtype)
        assert_rows(seen_rows[~hit], want[50:][~hit], bound[50:][~hit], what)
    else:
        q, k, v = split(x, h, hkv, dh)
        seen = torch.ones(100, 100, dtype=torch.bool, device="cuda").tril()
        vc = torch.nan_to_num(v, nan=0.0, posinf=0.0)
        want, bound = attention(q[off[1]:off[2]], k[off[1]:off[2]], vc[off[1]:off[2]], seen, 0.1, dtype)
        mine = got[off[1]:off[2]].reshape(-1, h, dh)
        cols = [c for c in range(dh) if c != 3]
        assert_rows(mine[:50], want[:50], bound[:50], what)
        assert_rows(mine[50:][:, :, cols], want[50:][:, :, cols], bound[50:][:, :, cols], what)
        hit = mine[50:, :, 3]
        assert bool(torch.isnan(hit).all() if "nan" in what else (hit == float("inf")).all())
    for b in (0, 2):
        q, k, v = split(x, h, hkv, dh)
        n = lens[b]
        seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        want, bound = attention(q[off[b]:off[b + 1]], k[off[b]:off[b + 1]], v[off[b]:off[b + 1]], seen, 0.1, dtype)
        assert_rows(got[off[b]:off[b + 1]].reshape(n, h, dh), want, bound, (what, b))


def test_streams_and_a_graph():
    """The same call on two streams at once, and captured and replayed with new inputs and offsets."""
    import torch
    h, hkv, dh = 4, 4, 64
    cases = [make(lens, h, hkv, dh, "f16", seed=i) for i, lens in enumerate(([200, 56], [10, 246]))]
    want = [run(x, off, rows, h, hkv, dh, "f16", True, 0.125) for x, off, rows in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [torch.full_like(w, 7.0) for w in want]
    offs = [torch.tensor(off, dtype=torch.int32, device="cuda") for _, off, _ in cases]
    torch.cuda.synchronize()
    for _ in range(4):
        for (x, off, rows), st, o, d in zip(cases, streams, outs, offs):
            run(x, off, rows, h, hkv, dh, "f16", True, 0.125, out=o, d_off=d, stream=st.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))

    x, off, rows = cases[0]
    xs, d, o = x.clone(), offs[0].clone(), torch.full_like(want[0], 7.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(xs, off, rows, h, hkv, dh, "f16", True, 0.125, out=o, d_off=d, stream=torch.cuda.current_stream().cuda_stream)
    for turn in range(4):
        src, off_t = cases[turn % 2][0], offs[turn % 2]
        xs.copy_(src)
        d.copy_(off_t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[turn % 2]), turn


def test_offsets_past_32_bits():
    """Rows whose distance from the first passes 2^32 bytes."""
    import torch
    h, dh, ld = 1, 32, 1 << 20
    rows = 2200
    x = torch.zeros(rows, ld, dtype=torch.float16, device="cuda")
    g = torch.Generator().manual_seed(2)
    x[:, :3 * dh] = torch.randn(rows, 3 * dh, generator=g).half().cuda()
    off = [0, 100, 2200]
    got = run(x, off, rows, h, 1, dh, "f16", True, 0.2)
    check(got, x[:, :3 * dh], off, h, 1, dh, "f16", True, 0.2)
