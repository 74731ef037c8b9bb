"""GPU: the paged key/value cache, nt_op_kv_append and nt_op_attn_paged, against float64."""
import numpy as np
import pytest

from tests.paged_util import Pages, assert_within, attend, attention_of_many, torch_dtype

pytestmark = pytest.mark.gpu

TYPES = [("f16", False), ("bf16", False), ("f32", False), ("f16", True)]


def _q(n, heads, d_head, dtype, seed, pad=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    wide = torch.full((n, heads * d_head + pad), float("nan"), dtype=torch_dtype(dtype))
    wide[:, :heads * d_head] = torch.randn(n, heads * d_head, generator=g).to(wide.dtype)
    return wide.cuda()[:, :heads * d_head].unflatten(1, (heads, d_head))


# ---- append ----------------------------------------------------------------------------
def _append_expected(pages, k, v, off, lens, n_rows):
    """The pools after the call, from the rows as the documentation places them."""
    import torch
    out = []
    for pool, x in ((pages.k, k), (pages.v, v)):
        p = pool.cpu().clone()
        x = x.cpu().view(k.shape[0], pages.kv_heads, pages.d_head)
        if pages.fp8:
            x = x.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        for b in range(len(lens)):
            lo, hi = (b, b + 1) if off is None else (off[b], off[b + 1])
            for i in range(lo, min(hi, n_rows)):
                pos = lens[b] - (hi - i)
                if pos < 0 or pos >= pages.max_pages * pages.page:
                    continue
                pid = int(pages.table_np[b, pos // pages.page])
                if 0 <= pid < pages.n_pages:
                    p[pid, :, pos % pages.page] = x[i]
        out.append(p)
    return out


def _append(pages, x, off, n_rows, lens=None):
    import torch
    from paper_2109_08008_amd import nt
    w = pages.kv_heads * pages.d_head
    d_off = None if off is None else torch.tensor(off, dtype=torch.int32, device="cuda")
    eb = x.element_size()
    nt.nt_op_kv_append(pages.cache, x.data_ptr() + w * eb, x.data_ptr() + 2 * w * eb, x.stride(0),
                       None if d_off is None else d_off.data_ptr(), (pages.lens if lens is None else lens).data_ptr(),
                       len(pages.lens_list), n_rows)
    torch.cuda.synchronize()


def _same(a, b):
    """Bitwise (NaN cells included)."""
    import torch
    as_int = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.cpu().view(as_int), b.cpu().view(as_int))


@pytest.mark.parametrize("dtype,fp8", TYPES)
@pytest.mark.parametrize("kv_heads,d_head,page", [(1, 32, 16), (3, 64, 16), (8, 64, 32), (5, 128, 256), (16, 128, 64)])
def test_append_places_rows(dtype, fp8, kv_heads, d_head, page):
    """Ragged new rows (none, one, more than a page), rows before the first and behind the last
    sequence, and every other cell left as it was, bit for bit."""
    import torch
    new = [0, 1, 37, 0, 2, 300, 16, 1]
    lens = [0, 1, 40, 9, 700, 300, 31, 257]
    off = np.concatenate([[2], 2 + np.cumsum(new)]).tolist()
    rows = off[-1] + 3
    pages = Pages(lens, kv_heads, d_head, page, dtype, fp8, seed=1)
    g = torch.Generator().manual_seed(5)
    w = kv_heads * d_head
    x = (torch.randn(rows, 3 * w + 16, generator=g) * 3).to(torch_dtype(dtype))
    x[5, :] = 1000.0            # E4M3 saturates
    x = x.cuda()
    want = _append_expected(pages, x[:, w:2 * w].contiguous(), x[:, 2 * w:3 * w].contiguous(), off, lens, rows)
    _append(pages, x, off, rows)
    assert _same(pages.k, want[0]) and _same(pages.v, want[1])


@pytest.mark.parametrize("dtype,fp8", TYPES)
@pytest.mark.parametrize("n", [1, 3, 64, 129, 5000])
def test_append_one_token_each(dtype, fp8, n):
    import torch
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 40, n).tolist()
    pages = Pages(lens, 2, 64, 16, dtype, fp8, seed=n)
    x = torch.randn(n, 3 * 128, generator=torch.Generator().manual_seed(n)).to(torch_dtype(dtype)).cuda()
    want = _append_expected(pages, x[:, 128:256].contiguous(), x[:, 256:].contiguous(), None, lens, n)
    _append(pages, x, None, n)
    assert _same(pages.k, want[0]) and _same(pages.v, want[1])


def test_append_rounds_every_fp16_value():
    """All 65536 fp16 codes through an FP8 cache: the library's E4M3 rounding (nearest even,
    saturating at 448, NaN to 0x7F), restated here on the exact values."""
    import torch
    from paper_2109_08008_amd import nt
    bits = np.arange(65536, dtype=np.uint16)
    x = bits.view(np.float16).astype(np.float64)
    nan = np.isnan(x)
    a = np.minimum(np.where(nan, 0.0, np.abs(x)), 448.0)
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    a = np.minimum(np.rint(a / step) * step, 448.0)
    want = torch.from_numpy(np.where(np.signbit(x), -a, a).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    want = np.where(nan, 0x7F, want)
    pages = Pages([512], 1, 128, 256, "f16", fp8=True, seed=1)
    rows = torch.from_numpy(bits.view(np.int16).reshape(512, 128).copy()).cuda()
    off = torch.tensor([0, 512], dtype=torch.int32, device="cuda")
    nt.nt_op_kv_append(pages.cache, rows.data_ptr(), rows.data_ptr(), 128, off.data_ptr(), pages.lens.data_ptr(), 1, 512)
    for pool in (pages.k, pages.v):
        got = torch.cat([pool[int(pages.table_np[0, j]), 0] for j in (0, 1)]).cpu().numpy().reshape(-1)
        got = np.where(nan & (got == 0xFF), 0x7F, got)      # a NaN's sign is no matter
        np.testing.assert_array_equal(got, want)


def test_append_many_sequences_search():
    """More sequences than two rounds of 64 probes, most without a row."""
    import torch
    n = 9000
    rng = np.random.default_rng(3)
    new = (rng.random(n) < 0.05).astype(int) * rng.integers(1, 5, n)
    new[[0, n - 1]] = [2, 3]
    lens = (new + rng.integers(0, 3, n)).tolist()
    off = np.concatenate([[0], np.cumsum(new)]).tolist()
    pages = Pages(lens, 1, 32, 16, "bf16", seed=2)
    x = torch.randn(off[-1], 96, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    want = _append_expected(pages, x[:, 32:64].contiguous(), x[:, 64:].contiguous(), off, lens, off[-1])
    _append(pages, x, off, off[-1])
    assert _same(pages.k, want[0]) and _same(pages.v, want[1])


def test_append_leaves_out_what_has_no_place():
    """Holes and page ids out of range, positions past the table and below 0, an inactive slot,
    offsets that claim more rows than there are."""
    import torch
    lens = [20, 33, 16, 5, 64]
    pages = Pages(lens, 2, 32, 16, "f16", seed=4)
    table = pages.table_np.copy()
    table[0, 1] = -1
    table[1, 2] = pages.n_pages
    table[1, 0] = 2 ** 31 - 1
    pages.retable(table)
    given = [20, 33, 200, -4, 64]      # past max_pages * page_len = 64; below 0
    pages.lens = torch.tensor(given, dtype=torch.int32, device="cuda")
    off = [0, 20, 53, 60, 62, 126]
    rows = 100                         # fewer than off says
    x = torch.randn(rows, 192, generator=torch.Generator().manual_seed(1)).half().cuda()
    want = _append_expected(pages, x[:, 64:128].contiguous(), x[:, 128:].contiguous(), off, given, rows)
    _append(pages, x, off, rows)
    assert _same(pages.k, want[0]) and _same(pages.v, want[1])


# ---- attention -------------------------------------------------------------------------
EDGE = [1, 15, 16, 17, 31, 32, 33, 0, 64, 65, 127, 128, 129, 191, 255, 256, 257]


@pytest.mark.parametrize("dtype,fp8", TYPES)
@pytest.mark.parametrize("d_head", [32, 64, 128])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_attention_at_the_edges(dtype, fp8, d_head, page):
    """Lengths on both sides of every block, tile and page edge; empty rows; everything that no
    sequence holds is NaN."""
    pages = Pages(EDGE, 2, d_head, page, dtype, fp8, seed=d_head + page).fill(1)
    q = _q(len(EDGE), 4, d_head, dtype, 2, pad=8)
    got = attend(pages, q, d_head ** -0.5)
    want, bound = pages.attention(q, d_head ** -0.5)
    assert_within(got, want, bound)
    assert (got[EDGE.index(0)] == 0).all()


@pytest.mark.parametrize("dtype,fp8", TYPES)
@pytest.mark.parametrize("kv_heads,group", [(1, 1), (3, 1), (2, 3), (1, 8), (2, 16), (1, 17), (1, 33), (2, 40)])
def test_attention_shared_heads(dtype, fp8, kv_heads, group):
    pages = Pages([70, 3, 200], kv_heads, 64, 16, dtype, fp8, seed=group).fill(3)
    q = _q(3, kv_heads * group, 64, dtype, 4)
    got = attend(pages, q, 0.125)
    assert_within(got, *pages.attention(q, 0.125))


@pytest.mark.parametrize("dtype,fp8", TYPES)
@pytest.mark.parametrize("d_head", [32, 64, 128])
@pytest.mark.parametrize("lens", [[5000], [1, 3000, 0, 769], [2049, 2048, 2047]])
def test_attention_split_over_the_length(dtype, fp8, d_head, lens):
    """Few tasks: the length is divided over workgroups and joined."""
    from paper_2109_08008_amd import nt
    pages = Pages(lens, 1, d_head, 64, dtype, fp8, seed=sum(lens)).fill(5)
    assert nt.nt_op_attn_paged_workspace(pages.cache, 2, len(lens), max(lens)) > 0
    q = _q(len(lens), 2, d_head, dtype, 6)
    got = attend(pages, q, d_head ** -0.5)
    assert_within(got, *pages.attention(q, d_head ** -0.5))


@pytest.mark.parametrize("n_seqs,max_len", [(1, 130), (1, 4096), (40, 300), (700, 260)])
def test_attention_lengths_below_the_bound(n_seqs, max_len):
    """max_len may be far above the lengths (parts with nothing to do), or below the table's
    reach; lengths above it are cut there."""
    rng = np.random.default_rng(n_seqs)
    lens = rng.integers(0, min(max_len, 300), n_seqs).tolist()
    lens[0] = 129
    pages = Pages(lens, 2, 32, 32, "f16", seed=9, extra_pages=max_len // 32).fill(7)
    q = _q(n_seqs, 2, 32, "f16", 8)
    got = attend(pages, q, 0.2, max_len=max_len)
    assert_within(got, *pages.attention(q, 0.2))
    got = attend(pages, q, 0.2, max_len=100)
    assert_within(got, *pages.attention(q, 0.2, lens=[min(n, 100) for n in lens]))


@pytest.mark.parametrize("dtype,fp8", TYPES)
@pytest.mark.parametrize("lens", [[200, 64, 40, 96], [3000, 64, 40, 2000]])
def test_attention_over_holes(dtype, fp8, lens):
    """Entries outside the pool are left out: a first page, a middle one, a last one, all; and
    lengths past the table's end or below 0."""
    import torch
    pages = Pages(lens, 1, 64, 16, dtype, fp8, seed=11).fill(9)
    table = pages.table_np.copy()
    table[0, [0, 5, 6, 12]] = [-1, pages.n_pages, -7, 2 ** 31 - 1]
    table[1] = -1
    table[2, :2] = -1
    pages.retable(table)
    pages.lens_list = [lens[0], 64, 40, -3]
    pages.lens = torch.tensor([lens[0] + 0, 64, 40, -3], dtype=torch.int32, device="cuda")
    q = _q(4, 2, 64, dtype, 10)
    got = attend(pages, q, 0.125, max_len=max(lens))
    assert_within(got, *pages.attention(q, 0.125))
    assert (got[1] == 0).all() and (got[3] == 0).all()
    pages.lens = torch.tensor([2 ** 31 - 1, 64, 40, -2 ** 31], dtype=torch.int32, device="cuda")   # cut at max_len
    again = attend(pages, q, 0.125, max_len=lens[0])
    assert torch.equal(again, got) or lens[0] < max(lens)


@pytest.mark.parametrize("n", [1, 700, 3000])
def test_attention_over_nothing(n):
    """No positions anywhere, max_len 0 and not: zeros."""
    import torch
    pages = Pages([0] * n, 1, 64, 16, "bf16", seed=1, extra_pages=300)
    q = _q(n, 2, 64, "bf16", 1)
    for max_len in (0, 16, 4800):
        assert (attend(pages, q, 0.125, max_len=max_len) == 0).all()
    pages.lens.fill_(-2 ** 31)
    assert (attend(pages, q, 0.125, max_len=100) == 0).all()


def test_attention_leaves_other_rows():
    """Rows behind the last sequence, and what lies between the rows, stay as they were."""
    import torch
    for lens in ([40, 3], [4000, 3]):
        pages = Pages(lens, 1, 64, 16, "f16", seed=1).fill(1)
        q = _q(5, 2, 64, "f16", 1)
        wide = torch.full((5, 2 * 64 + 24), 7.0, dtype=torch.float16, device="cuda")
        out = wide[:, :128].unflatten(1, (2, 64))
        attend(pages, q, 0.125, n_seqs=2, out=out)
        assert_within(out[:2], *pages.attention(q[:2], 0.125))
        assert (wide[2:] == 7).all() and (wide[:, 128:] == 7).all()


def test_attention_extreme_scores():
    """Scores far apart (all weight on one key), equal scores, large values, infinite values at
    positions that are not attended to, and an infinite value that is."""
    import torch
    pages = Pages([300, 300, 50], 1, 64, 16, "f16", seed=3).fill(3)
    for b, j in ((0, 17), (1, 299)):
        pages.k[int(pages.table_np[b, j // 16]), 0, j % 16] = 60.0
    pages.k[[int(x) for x in pages.table_np[2, :4]]] = 0.0
    pages.v[int(pages.table_np[2, 3]), 0, 2:] = float("inf")      # positions 50..: behind the length
    q = _q(3, 1, 64, "f16", 3).abs()
    q[0] = 10.0
    got = attend(pages, q, 1.0)
    want, bound = pages.attention(q, 1.0)
    assert_within(got, want, bound)
    pages.v[int(pages.table_np[2, 0]), 0, 5, 9] = float("inf")
    got = attend(pages, q, 1.0)
    assert got[2, 0, 9] == float("inf") and torch.isfinite(got[2, 0, :9]).all() and torch.isfinite(got[2, 0, 10:]).all()


def test_attention_over_shared_pages():
    """Hypotheses whose rows of the table name the same pages for a common prefix."""
    pages = Pages([90, 90, 90], 2, 32, 16, "bf16", seed=6).fill(6)
    table = pages.table_np.copy()
    table[1, :5] = table[0, :5]
    table[2, :3] = table[0, :3]
    pages.retable(table)
    pages.fill(8)
    q = _q(3, 2, 32, "bf16", 6)
    got = attend(pages, q, 0.3)
    assert_within(got, *pages.attention(q, 0.3))


def test_attention_past_32_bit_offsets():
    """Pages beyond 2^32 elements (and 2^33 bytes) of a pool, written and read."""
    import torch
    from paper_2109_08008_amd import nt
    page, hkv, dh = 256, 16, 128
    n_pages = (1 << 32) // (page * hkv * dh) + 3
    k = torch.empty(n_pages, hkv, page, dh, dtype=torch.float16, device="cuda")
    v = torch.empty_like(k)
    lens = [300, 2]
    small = Pages(lens, hkv, dh, page, "f16", seed=2)
    for pool in (k, v):
        pool[n_pages - 4:] = float("nan")
    table = np.array([[n_pages - 1, n_pages - 3], [n_pages - 2, -1]], dtype=np.int32)
    d_table = torch.from_numpy(table).cuda()
    cache = nt.kv_pages("f16", hkv, dh, page, n_pages, 2, k.data_ptr(), v.data_ptr(), d_table.data_ptr())
    w = hkv * dh
    x = torch.randn(302, 3 * w, generator=torch.Generator().manual_seed(2)).half().cuda()
    off = torch.tensor([0, 300, 302], dtype=torch.int32, device="cuda")
    nt.nt_op_kv_append(cache, x.data_ptr() + 2 * w, x.data_ptr() + 4 * w, 3 * w, off.data_ptr(), small.lens.data_ptr(), 2, 302)
    # the same through a small pool
    _append(small, x, [0, 300, 302], 302)
    for b, j in ((0, 0), (0, 1), (1, 0)):
        assert _same(k[int(table[b, j])], small.k[int(small.table_np[b, j])])
        assert _same(v[int(table[b, j])], small.v[int(small.table_np[b, j])])
    q = _q(2, hkv, dh, "f16", 1)
    want = attend(small, q, 0.09)
    out = torch.empty_like(want)
    need = nt.nt_op_attn_paged_workspace(cache, hkv, 2, 300)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    nt.nt_op_attn_paged(cache, q.data_ptr(), w, hkv, small.lens.data_ptr(), 2, 300, 0.09, out.data_ptr(), w, ws.data_ptr(), need)
    assert _same(out, want)


@pytest.mark.parametrize("lens", [[30, 31, 32], [1500, 2, 700]])
def test_step_captured_and_replayed(lens):
    """Append and attention captured into one graph and replayed over new rows and lengths; eager
    work of the same kind between the replays; every replay equals the eager result."""
    import torch
    page, hkv, heads, dh, n = 32, 2, 4, 64, 3
    steps = 4
    cap = max(lens) + steps
    pages = Pages([cap] * n, hkv, dh, page, "f16", seed=1)
    eager = Pages([cap] * n, hkv, dh, page, "f16", seed=1)
    for p in (pages, eager):
        p.fill(2)
    w = hkv * dh
    x = torch.empty(n, 3 * w, dtype=torch.float16, device="cuda")
    q = _q(n, heads, dh, "f16", 1)
    cur = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = torch.empty(n, heads, dh, dtype=torch.float16, device="cuda")
    from paper_2109_08008_amd import nt
    need = nt.nt_op_attn_paged_workspace(pages.cache, heads, n, cap)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")

    def step(p, o, work):
        nt.nt_op_kv_append(p.cache, x.data_ptr() + 2 * w, x.data_ptr() + 4 * w, 3 * w, None, cur.data_ptr(), n, n)
        nt.nt_op_attn_paged(p.cache, q.data_ptr(), heads * dh, heads, cur.data_ptr(), n, cap, 0.125, o.data_ptr(), heads * dh,
                            work.data_ptr(), work.numel())

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(pages, out, ws)
    for t in range(steps):
        cur.fill_(0)
        cur += torch.tensor(lens, dtype=torch.int32, device="cuda") + t
        x.copy_(torch.randn(n, 3 * w, generator=torch.Generator().manual_seed(t)).half())
        graph.replay()
        want = torch.empty_like(out)
        step(eager, want, torch.empty_like(ws))
        torch.cuda.synchronize()
        assert _same(out, want) and _same(pages.k, eager.k) and _same(pages.v, eager.v)


def test_two_streams_with_their_own_workspaces():
    import torch
    pages = Pages([3000, 800], 2, 64, 32, "bf16", seed=4).fill(4)
    q = [_q(2, 4, 64, "bf16", s) for s in (1, 2)]
    want = [attend(pages, x, 0.125) for x in q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in q]
    got = [torch.empty_like(want[0]) for _ in range(6)]
    ws = [torch.empty(1 << 22, dtype=torch.uint8, device="cuda") for _ in q]
    for i in range(6):
        attend(pages, q[i % 2], 0.125, out=got[i], ws=ws[i % 2], stream=streams[i % 2].cuda_stream)
    torch.cuda.synchronize()
    for i in range(6):
        assert _same(got[i], want[i % 2])


def test_undersized_workspace_is_reported():
    import torch
    from paper_2109_08008_amd import nt
    pages = Pages([4000], 1, 64, 16, "f16", seed=1).fill(1)
    q = _q(1, 1, 64, "f16", 1)
    need = nt.nt_op_attn_paged_workspace(pages.cache, 1, 1, 4000)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for ptr, size in ((ws.data_ptr(), need - 1), (None, need)):
        with pytest.raises(nt.NTError) as e:
            nt.nt_op_attn_paged(pages.cache, q.data_ptr(), 64, 1, pages.lens.data_ptr(), 1, 4000, 0.1, q.data_ptr(), 64, ptr, size)
        assert e.value.status == nt.NT_E_WORKSPACE and str(need) in e.value.message


# ---- how exactly the probabilities enter the second product -------------------------------
def _set(pool, index, value, fp8):
    """pool[index] = value, in the cache's type."""
    import torch
    x = torch.as_tensor(value, dtype=torch.float32)
    pool[index] = (x.to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else x.to(pool.dtype)).to(pool.device)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d_head", [32, 64, 128])
@pytest.mark.parametrize("n,length", [(1, 60000), (64, 8000), (2048, 250)])
def test_attention_keeps_the_tail_of_a_dominant_key(fp8, d_head, n, length):
    """One key far above thousands of equal ones, whose values alone are not zero: the output is the
    others' weight.  A probability is off by at most half a step of fp16 (2^-11 of itself) down to
    2^-28 of the largest and by half of fp16's least value below that, 2^-39 of the largest."""
    import torch
    pages = Pages([length] * n, 1, d_head, 64, "f16", fp8, seed=3)
    q = torch.zeros(n, 1, d_head, dtype=torch.float16, device="cuda")
    q[:, :, 0] = 1.0
    for at in (0, length - 1):
        first = pages.table[:, at // 64].long()
        for gap in (9.0, 11.0, 18.0, 20.0, 24.0):      # exact in every type
            _set(pages.k, slice(None), 0.0, fp8)
            _set(pages.v, slice(None), 1.0, fp8)
            _set(pages.k, (first, 0, at % 64, 0), gap, fp8)
            _set(pages.v, (first, 0, at % 64), 0.0, fp8)
            got = attend(pages, q, 1.0)
            e = np.exp(-gap)
            mass = (length - 1) * e / (1 + (length - 1) * e)
            # (scores of one product are exact but for the scaling and the exponential's 2^-21; sums of
            # `length` terms; the output's half step, or half of fp16's least value)
            tol = mass * (2.0 ** -11 + 2.0 ** -11 + 4 * gap * 2.0 ** -24 + 2.0 ** -20 + length * 2.0 ** -24) + (
                length * 2.0 ** -39 + 2.0 ** -25)
            off = (got.double() - mass).abs().max().item()
            assert off <= tol, (at, gap, mass, off, tol)


# What a probability may be off by in P.V, of itself and of the largest: two terms of 16 bits hold it to
# 2^-19 (fp16; its least value being 2^-38 of the largest probability) and 2^-16 (bf16).
P_REL = {"f16": 2.0 ** -19, "bf16": 2.0 ** -16, "f32": 0.0}
P_ABS = {"f16": 2.0 ** -38, "bf16": 0.0, "f32": 0.0}


@pytest.mark.parametrize("dtype,fp8", TYPES)
@pytest.mark.parametrize("d_head", [32, 64, 128])
@pytest.mark.parametrize("n,length", [(3, 21), (1, 3000), (2100, 200)])
def test_attention_of_values_that_cancel(dtype, fp8, d_head, n, length):
    """A third of the keys at a score above the others' by about log 2, values of opposite sign: the
    output is what is left of sums a thousand times as large, so that a step of P would show."""
    import torch
    pages = Pages([length] * n, 1, d_head, 16, dtype, fp8, seed=5)
    gaps = [0.625, 0.6875, 0.703125, 0.75, 1.0, 0.3125]
    q = torch.zeros(n, len(gaps), d_head, dtype=torch_dtype(dtype), device="cuda")
    q[:, :, 0] = torch.tensor(gaps, dtype=q.dtype)
    third = (torch.arange(16 * pages.max_pages) % 3 == 0).float().view(pages.max_pages, 16)
    value = torch.where(third[..., None] > 0, torch.ones(d_head), -(torch.arange(d_head) % 16 + 1) / 16.0)
    for j in range(pages.max_pages):
        at = pages.table[:, j].long()
        _set(pages.k, (at, 0), 0.0, fp8)
        _set(pages.k, (at, 0, slice(None), 0), third[j], fp8)
        _set(pages.v, (at, 0), value[j], fp8)
    got = attend(pages, q, 1.0)
    assert_within(got, *attention_of_many(pages, q, 1.0, P_REL[dtype], P_ABS[dtype]))


@pytest.mark.parametrize("dtype,fp8", TYPES)
@pytest.mark.parametrize("d_head", [32, 64, 128])
@pytest.mark.parametrize("lens", [EDGE, [3000, 1, 0, 769, 2049]])
def test_attention_rounds_the_output_only(dtype, fp8, d_head, lens):
    """Random keys and values: half a step of the output, and fp32's roundings."""
    pages = Pages(lens, 2, d_head, 32, dtype, fp8, seed=d_head).fill(21)
    q = _q(len(lens), 6, d_head, dtype, 22)
    got = attend(pages, q, d_head ** -0.5)
    assert_within(got, *attention_of_many(pages, q, d_head ** -0.5, P_REL[dtype], P_ABS[dtype]))


# ---- many short tasks, a wave each ------------------------------------------------------
def _fill_all(pages, seed):
    """Random cells at every held position, NaN everywhere else, all sequences at once."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    page = pages.page
    table = pages.table.long()
    counts = (torch.tensor(pages.lens_list, device="cuda")[:, None] - page * torch.arange(table.shape[1], device="cuda")).clamp(0, page)
    real = (table >= 0) & (table < pages.n_pages)
    held = torch.zeros(pages.n_pages, page, dtype=torch.bool, device="cuda")
    held[table[real]] = torch.arange(page, device="cuda") < counts[real][:, None]
    for pool in (pages.k, pages.v):
        x = torch.randn(pool.shape, generator=g, device="cuda")
        x = x.to(torch.float8_e4m3fn).view(torch.uint8) if pages.fp8 else x.to(pool.dtype)
        pool.copy_(torch.where(held[:, None, :, None], x, pool))
    return pages


@pytest.mark.parametrize("dtype,fp8", TYPES)
@pytest.mark.parametrize("d_head", [32, 64, 128])
@pytest.mark.parametrize("n,kv_heads,group,page,longest", [(2049, 1, 1, 16, 256), (683, 3, 3, 128, 256), (1025, 1, 17, 32, 256),
                                                           (347, 2, 33, 16, 129), (1030, 2, 1, 64, 40), (2203, 1, 4, 256, 17)])
def test_attention_of_many_short_tasks(dtype, fp8, d_head, n, kv_heads, group, page, longest):
    """2048 tasks (sequence, key head, block of 16 query heads) and more of up to 256 keys, which are a
    wave's each: lengths on both sides of every tile and page edge, none and negative ones, holes, more
    than one block of heads, a number of tasks that four does not divide; nothing between the rows or
    behind the last one changes."""
    import torch
    from paper_2109_08008_amd import nt
    tasks = n * kv_heads * ((group + 15) // 16)
    assert tasks >= 2048 and (n != 2049 or tasks % 4)
    rng = np.random.default_rng(n + d_head)
    lens = rng.integers(0, longest + 1, n)
    edge = [x for x in EDGE if x <= longest] + [longest]
    lens[rng.permutation(n)[:4 * len(edge)]] = np.tile(edge, 4)
    pages = _fill_all(Pages(lens.tolist(), kv_heads, d_head, page, dtype, fp8, seed=n), n)
    table = pages.table_np.copy()
    table[rng.random(table.shape) < 0.04] = rng.choice([-1, pages.n_pages, 2 ** 31 - 1, -2 ** 31])
    pages.retable(table)
    lens[7] = -3
    pages.lens_list = lens.tolist()
    pages.lens = torch.from_numpy(lens.astype(np.int32)).cuda()
    heads = kv_heads * group
    assert nt.nt_op_attn_paged_workspace(pages.cache, heads, n, longest) == 0
    q = _q(n, heads, d_head, dtype, 2, pad=8)
    wide = torch.full((n + 3, heads * d_head + 16), 7.0, dtype=q.dtype, device="cuda")
    out = wide[:, :heads * d_head].unflatten(1, (heads, d_head))
    attend(pages, q, d_head ** -0.5, max_len=longest, out=out)
    want, bound = attention_of_many(pages, q, d_head ** -0.5, P_REL[dtype], P_ABS[dtype])
    assert_within(out[:n], want, bound)
    assert (out[:n][torch.from_numpy(lens <= 0)] == 0).all()
    assert (wide[n:] == 7).all() and (wide[:, heads * d_head:] == 7).all()


# ---- appends of many and of wide rows -----------------------------------------------------
def _append_all(pages, x, off, lens):
    """_append_expected for many rows at once."""
    import torch
    w, page = pages.kv_heads * pages.d_head, pages.page
    off, lens = np.asarray(off), np.asarray(lens)
    seq = np.repeat(np.arange(len(lens)), np.diff(off))
    row = np.arange(off[0], off[-1])
    pos = lens[seq] - (off[seq + 1] - row)
    assert (pos >= 0).all() and (pos < pages.max_pages * page).all()
    at = torch.from_numpy(pages.table_np[seq, pos // page].astype(np.int64))
    slot = torch.from_numpy(pos % page)
    out = []
    for part, pool in ((1, pages.k), (2, pages.v)):
        new = x.cpu()[off[0]:off[-1], part * w:(part + 1) * w].reshape(-1, pages.kv_heads, pages.d_head)
        if pages.fp8:
            new = new.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        p = pool.cpu().clone()
        p[at, :, slot] = new
        out.append(p)
    return out


@pytest.mark.parametrize("dtype,fp8", TYPES)
@pytest.mark.parametrize("kv_heads,d_head,n,longest", [
    (1, 32, 1500, 401),       # 300 thousand narrow rows: several a wave in several turns
    (1, 64, 900, 301),        # the same of twice the width
    (5, 64, 300, 201),        # rows that no power of two of lanes covers, several turns a wave
    (16, 64, 400, 151),       # two turns a row, several rows a wave
    (17, 128, 90, 231),       # ends of rows inside a turn
    (40, 128, 12, 61)])       # rows past 8 KB: more turns than are under way at once
def test_append_of_many_and_wide_rows(dtype, fp8, kv_heads, d_head, n, longest):
    import torch
    rng = np.random.default_rng(n)
    new = rng.integers(0, longest, n)
    new[[0, 1, n - 1]] = [3, 0, longest]
    lens = new + rng.integers(0, 20, n)
    off = 1 + np.concatenate([[0], np.cumsum(new)])
    pages = Pages(lens.tolist(), kv_heads, d_head, 32, dtype, fp8, seed=n)
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(int(off[-1]) + 2, 3 * kv_heads * d_head, generator=g, device="cuda").to(torch_dtype(dtype))
    want = _append_all(pages, x, off, lens)
    _append(pages, x, off.tolist(), len(x))
    assert _same(pages.k, want[0]) and _same(pages.v, want[1])


@pytest.mark.parametrize("dtype,fp8", TYPES)
def test_append_of_equal_rows_to_a_shared_page(dtype, fp8):
    """Sequences that extend a page they share by the same token: that token's row."""
    import torch
    n, hkv, dh = 70, 3, 64
    pages = Pages([21] * n, hkv, dh, 16, dtype, fp8, seed=2)
    table = pages.table_np.copy()
    table[:, 1] = table[0, 1]
    pages.retable(table)
    x = torch.randn(1, 3 * hkv * dh, generator=torch.Generator().manual_seed(3)).to(torch_dtype(dtype)).cuda().repeat(n, 1)
    w = hkv * dh
    want = _append_expected(pages, x[:, w:2 * w].contiguous(), x[:, 2 * w:].contiguous(), None, pages.lens_list, n)
    _append(pages, x, None, n)
    assert _same(pages.k, want[0]) and _same(pages.v, want[1])
