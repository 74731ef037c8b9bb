"""GPU: nt_op_attn_tree, attention of several new tokens a sequence over a paged cache, against float64."""
import pytest

from tests.paged_util import Pages, attend, torch_dtype
from tests.rows_util import assert_rows, attention

pytestmark = pytest.mark.gpu


def trees(new, seed=0, own_bit=True):
    """Ancestor words of random trees, one list a sequence."""
    import random
    r = random.Random(seed)
    got = []
    for n in new:
        seen = []
        for i in range(n):
            p = r.randint(max(-1, i - 5), i - 1)
            seen.append((1 << i if own_bit else 0) | (seen[p] | (1 << p) if p >= 0 else 0))
        got.append(seen)
    return got


def run(pages, q, new, masks, scale, max_new=None, max_len=None, off=None, ws=None, out=None, stream=None, n_rows=None):
    import torch
    from paper_2109_08008_amd import nt
    n, heads = len(new), q.shape[1]
    rows = q.shape[0] if n_rows is None else n_rows
    max_new = max([0] + list(new)) if max_new is None else max_new
    max_len = max([0] + pages.lens_list) if max_len is None else max_len
    if off is None:
        off = torch.tensor([sum(new[:b]) for b in range(n + 1)], dtype=torch.int32, device=q.device)
    d_mask = None
    if masks is not None:
        words = [w - (1 << 64) if w >> 63 else w for m in masks for w in m]
        d_mask = torch.tensor(words + [0] * (rows - len(words)), dtype=torch.int64, device=q.device)
    if out is None:
        out = torch.full((q.shape[0], heads, pages.d_head), 7.0, dtype=q.dtype, device=q.device)
    need = nt.nt_op_attn_tree_workspace(pages.cache, heads, n, rows, max_new, max_len)
    if ws is None:
        ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device=q.device)   # NaN in every float
    nt.nt_op_attn_tree(pages.cache, q.data_ptr(), q.stride(0), heads, off.data_ptr() if off is not False else None,
                       d_mask.data_ptr() if d_mask is not None else None, pages.lens.data_ptr(), n, rows, max_new, max_len,
                       scale, out.data_ptr(), out.stride(0), ws.data_ptr() if need else None, need, stream)
    torch.cuda.synchronize()
    return out


def cells(pages, pool, b, n):
    """[n, kv_heads, d_head] of sequence b's positions in float64, and which of them have a page."""
    import torch
    pos = torch.arange(n)
    pid = torch.tensor([int(pages.table_np[b, p // pages.page]) for p in range(n)])
    held = (pid >= 0) & (pid < pages.n_pages)
    x = pool.view(torch.float8_e4m3fn) if pages.fp8 else pool
    x = x.cpu().to(torch.float64)[torch.where(held, pid, torch.zeros_like(pid)), :, pos % pages.page]
    return x.cuda(), held.cuda()


def check(got, pages, q, new, masks, scale, max_len=None):
    import torch
    row = 0
    for b, n in enumerate(new):
        if n == 0:
            continue
        length = pages.lens_list[b]
        base = length - n
        k, held = cells(pages, pages.k, b, length)
        v, _ = cells(pages, pages.v, b, length)
        pos = torch.arange(length, device="cuda")
        seen = torch.zeros(n, length, dtype=torch.bool, device="cuda")
        for i in range(n):
            seen[i] = pos < base
            for j in range(n):
                if base + j >= 0 and ((masks[b][i] >> j & 1) if masks is not None else j <= i):
                    seen[i, base + j] = True
        seen &= held
        if max_len is not None:
            seen &= pos < max_len
        want, bound = attention(q[row:row + n].double(), k, v, seen, scale, pages.dtype)
        assert_rows(got[row:row + n], want, bound, (b, n, length))
        row += n
    assert bool((got[row:] == 7.0).all()), "rows of no sequence were written"


def queries(rows, heads, d_head, dtype, seed=1, behind=2):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows + behind, heads, d_head, generator=g)
    x[rows:] = float("nan")
    return x.to(torch_dtype(dtype)).cuda()


CONFIGS = [("f16", False), ("f16", True), ("bf16", False), ("f32", False)]


@pytest.mark.parametrize("dtype,fp8", CONFIGS)
@pytest.mark.parametrize("group", [1, 3, 8])
@pytest.mark.parametrize("new", [[1, 1, 1], [8, 3, 0, 5], [64, 1, 33, 24]], ids=str)
@pytest.mark.parametrize("tree", [True, False])
def test_trees_and_chains(tree, new, group, dtype, fp8):
    hkv, dh = 2, 64
    lens = [n + c for n, c in zip(new, [0, 45, 200, 131])]
    pages = Pages(lens, hkv, dh, 16, dtype, fp8, seed=3).fill(4)
    q = queries(sum(new), hkv * group, dh, dtype)
    masks = trees(new) if tree else None
    check(run(pages, q, new, masks, dh ** -0.5), pages, q, new, masks, dh ** -0.5)


@pytest.mark.parametrize("dtype,fp8", CONFIGS)
@pytest.mark.parametrize("d_head", [32, 64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_heads_and_pages(page, d_head, dtype, fp8):
    new = [7, 20]
    pages = Pages([150, 333], 1, d_head, page, dtype, fp8, seed=page).fill(5)
    for group in (2, 5):
        q = queries(27, group, d_head, dtype, seed=group)
        masks = trees(new, seed=page)
        check(run(pages, q, new, masks, 0.1), pages, q, new, masks, 0.1)


@pytest.mark.parametrize("dtype,fp8", CONFIGS)
@pytest.mark.parametrize("group,new", [(1, 4), (4, 8), (4, 64)])
def test_long_caches_are_cut_and_joined(group, new, dtype, fp8):
    from paper_2109_08008_amd import nt
    lens, news = [5003, 700, new, 1], [new, 1, new, 1]
    pages = Pages(lens, 1, 64, 64, dtype, fp8, seed=6).fill(7)
    rows = sum(news)
    assert nt.nt_op_attn_tree_workspace(pages.cache, group, 4, rows, new, max(lens)) > 0
    q = queries(rows, group, 64, dtype)
    for masks in (trees(news, 2), None):
        check(run(pages, q, news, masks, 0.125, n_rows=rows), pages, q, news, masks, 0.125)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_pieces_of_prompts(dtype):
    new = [300, 1, 129, 77]
    lens = [300, 400, 1000, 80]
    pages = Pages(lens, 2, 64, 32, dtype, seed=8).fill(9)
    q = queries(sum(new), 6, 64, dtype)
    check(run(pages, q, new, None, 0.125), pages, q, new, None, 0.125)


def test_rows_that_see_nothing_are_zero():
    """A first token whose mask is empty, without context; and masks without the row's own bit."""
    import torch
    new, lens = [5, 4], [5, 40]
    pages = Pages(lens, 1, 64, 16, "f16", seed=1).fill(2)
    q = queries(9, 2, 64, "f16")
    masks = trees(new, own_bit=False)
    masks[0][0] = 0
    masks[0][3] = 0
    got = run(pages, q, new, masks, 0.125)
    check(got, pages, q, new, masks, 0.125)
    assert bool((got[0] == 0).all()) and bool((got[3] == 0).all())
    assert bool(torch.isfinite(got[:9]).all())


@pytest.mark.parametrize("dtype,fp8", CONFIGS)
def test_holes_are_left_out(dtype, fp8):
    new, lens = [6, 6], [100, 260]
    pages = Pages(lens, 1, 64, 16, dtype, fp8, seed=2).fill(3)
    table = pages.table_np.copy()
    table[0, 2] = -1
    table[0, 6] = pages.n_pages          # the last page, with new tokens
    table[1, 0] = 2 ** 31 - 1
    table[1, 9] = -7
    pages.retable(table)
    q = queries(12, 3, 64, dtype)
    masks = trees(new, 5)
    check(run(pages, q, new, masks, 0.2), pages, q, new, masks, 0.2)
    check(run(pages, q, new, None, 0.2), pages, q, new, None, 0.2)


@pytest.mark.parametrize("group", [1, 4, 16])
def test_positions_past_max_len_are_not_read(group):
    new, lens = [9, 9], [50, 300]
    pages = Pages(lens, 1, 64, 16, "bf16", seed=4).fill(5)
    q = queries(18, group, 64, "bf16")
    masks = trees(new, 6)
    for limit in (45, 100, 296):
        check(run(pages, q, new, masks, 0.125, max_len=limit), pages, q, new, masks, 0.125, max_len=limit)


def test_rows_past_max_new_are_not_written():
    import torch
    new, lens = [9, 3], [60, 70]
    pages = Pages(lens, 1, 64, 16, "f16", seed=4).fill(5)
    q = queries(12, 2, 64, "f16")
    got = run(pages, q, new, None, 0.125, max_new=4)
    assert bool((got[4:9] == 7.0).all()) and bool(torch.isfinite(got).all())


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("max_new", [1, 4, 17])
def test_rows_up_to_max_new_are_the_same(max_new, tree):
    """Where a sequence has more new tokens than max_new those before that see what they saw."""
    import torch
    new, lens = [20, 3, 40], [60, 70, 300]
    pages = Pages(lens, 1, 64, 16, "f16", seed=4).fill(5)
    q = queries(63, 2, 64, "f16")
    masks = trees(new, 9) if tree else None
    whole = run(pages, q, new, masks, 0.125)
    check(whole, pages, q, new, masks, 0.125)
    got = run(pages, q, new, masks, 0.125, max_new=max_new)
    row = 0
    for n in new:
        m = min(n, max_new)
        assert bool((got[row + m:row + n] == 7.0).all())
        got[row + m:row + n] = whole[row + m:row + n]
        row += n
    check(got, pages, q, new, masks, 0.125)


def test_offsets_that_fall():
    """Offsets below 0, past the rows or falling write no row outside the buffers, and those of other
    sequences are as without them."""
    import torch
    pages = Pages([60, 70, 80], 1, 64, 16, "f16", seed=4).fill(5)
    q = queries(12, 2, 64, "f16", behind=4)
    whole = run(pages, q, [0, 0, 5], None, 0.125)
    for bad in ([-2 ** 31, -2 ** 31, 0, 5], [2 ** 31 - 1, -2 ** 31, 0, 5], [12, 2 ** 31 - 1, 0, 5]):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        guard = torch.full((32, 2, 64), 7.0, dtype=torch.float16, device="cuda")
        got = run(pages, q, [0, 0, 0], None, 0.125, max_new=5, max_len=80, off=off, out=guard[8:24], n_rows=12)
        assert torch.equal(got[:5], whole[:5]), bad
        assert bool((guard[:8] == 7.0).all()) and bool((guard[20:] == 7.0).all()), bad


@pytest.mark.parametrize("dtype,fp8", CONFIGS)
@pytest.mark.parametrize("what", ["value", "key"])
@pytest.mark.parametrize("new", [6, 40])
def test_numbers_stay_with_the_rows_that_see_them(new, what, dtype, fp8):
    """A drafted token whose key or value holds a NaN: its siblings do not notice."""
    import torch
    pages = Pages([70, 90], 1, 64, 16, dtype, fp8, seed=9).fill(1)
    news = [new, new]
    masks = [[1 << i for i in range(new)] for _ in news]        # new tokens that see the context and themselves
    base = 70 - new
    pid = int(pages.table_np[0, (base + 2) // 16])
    pool = pages.v if what == "value" else pages.k
    pool[pid, 0, (base + 2) % 16, 5] = 0x7F if fp8 else float("nan")
    q = queries(2 * new, 2, 64, dtype)
    got = run(pages, q, news, masks, 0.125)
    mine = got[2]
    assert bool(torch.isnan(mine[:, 5]).all())
    if what == "key":
        assert bool(torch.isnan(mine).all())
    keep = [i for i in range(2 * new) if i != 2]
    pool[pid, 0, (base + 2) % 16, 5] = 0
    clean = run(pages, q, news, masks, 0.125)
    check(clean, pages, q, news, masks, 0.125)
    got[2] = clean[2]
    check(got, pages, q, news, masks, 0.125)
    assert bool(torch.isfinite(got[keep]).all())


def test_one_new_token_without_offsets_is_what_attn_paged_gives():
    import torch
    lens = [1, 40, 333, 1200]
    for dtype, tol in (("f32", 2e-5), ("f16", 4e-3), ("bf16", 3e-2)):
        pages = Pages(lens, 2, 64, 32, dtype, seed=1).fill(2)
        q = queries(4, 8, 64, dtype, behind=0)
        got = run(pages, q, [1] * 4, None, 0.125, off=False)
        check(got, pages, q, [1] * 4, None, 0.125)
        assert float((got.float() - attend(pages, q, 0.125).float()).abs().max()) < tol
        assert bool(torch.isfinite(got).all())


def test_many_sequences():
    """More sequences than the lanes of a wave, several row blocks, cut lengths."""
    n = 150
    new = [(i * 37) % 20 for i in range(n)]
    lens = [max(new[i], (i * 7919) % 900) for i in range(n)]
    pages = Pages(lens, 1, 32, 64, "f16", seed=3).fill(4)
    q = queries(sum(new), 4, 32, "f16")
    masks = trees(new, 8)
    check(run(pages, q, new, masks, 0.18), pages, q, new, masks, 0.18)


@pytest.mark.parametrize("dtype,fp8", CONFIGS)
@pytest.mark.parametrize("heads", [1, 3, 4])
@pytest.mark.parametrize("new", [3, 40])
def test_parts_of_lengths(new, heads, dtype, fp8):
    """Lengths around a half and a whole of the 512 keys that a part has at least, uncut, in two and in many."""
    lens = [3000, 1, 511, 512, 513, 767, 768, 769, 1024, 1279, 1280, 1281, 2999]
    news = [min(new, n) for n in lens]
    pages = Pages(lens, 1, 32, 64, dtype, fp8, seed=heads).fill(4)
    q = queries(sum(news), heads, 32, dtype)
    for masks in (trees(news, 5), None):
        check(run(pages, q, news, masks, 0.18), pages, q, news, masks, 0.18)


def test_a_length_below_the_new_tokens():
    """Lengths that do not hold all new tokens (the first of them have no position)."""
    new = [6, 6]
    pages = Pages([4, 20], 1, 64, 16, "f16", seed=3).fill(4)
    q = queries(12, 2, 64, "f16")
    masks = trees(new, 3)
    check(run(pages, q, new, masks, 0.125), pages, q, new, masks, 0.125)
    check(run(pages, q, new, None, 0.125), pages, q, new, None, 0.125)


def test_a_graph_of_cut_lengths():
    """Captured with a workspace of its own; lengths, masks and queries change between replays, and eager
    calls with another workspace run between them."""
    import torch
    from paper_2109_08008_amd import nt
    new = [5, 12]
    pages = Pages([3000, 1500], 1, 64, 64, "f16", seed=2).fill(3)
    full = pages.lens.clone()
    q = queries(17, 4, 64, "f16", behind=0)
    xs = q.clone()
    need = nt.nt_op_attn_tree_workspace(pages.cache, 4, 2, 17, 12, 3000)
    assert need > 0
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    off = torch.tensor([0, 5, 17], dtype=torch.int32, device="cuda")
    mask = torch.zeros(17, dtype=torch.int64, device="cuda")
    out = torch.full((17, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        nt.nt_op_attn_tree(pages.cache, xs.data_ptr(), 256, 4, off.data_ptr(), mask.data_ptr(), pages.lens.data_ptr(), 2, 17,
                           12, 3000, 0.125, out.data_ptr(), 256, ws.data_ptr(), need,
                           torch.cuda.current_stream().cuda_stream)
    for turn in range(4):
        lens = [3000 - 700 * turn, 1500 - 11 * turn]
        pages.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        pages.lens_list = lens
        masks = trees(new, turn)
        mask.copy_(torch.tensor([w for m in masks for w in m]))
        xs.copy_(q * (1 + turn))
        eager = run(pages, xs, new, masks, 0.125, max_len=3000)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), turn
        check(out, pages, xs, new, masks, 0.125)
    assert int(full[0]) == 3000


@pytest.mark.parametrize("dtype,fp8", CONFIGS)
@pytest.mark.parametrize("d_head", [32, 64, 128])
def test_many_short_sequences(d_head, dtype, fp8):
    """More tasks of few rows than fit the GPU at once; lengths around a tile's 32 and 64 keys."""
    n = 130
    new = [(i * 37) % 6 for i in range(n)]
    lens = [max(new[i], (i * 7919) % 140) for i in range(n)]
    pages = Pages(lens, 8, d_head, 16, dtype, fp8, seed=3).fill(4)
    q = queries(sum(new), 8, d_head, dtype)
    masks = trees(new, 8)
    check(run(pages, q, new, masks, 0.18), pages, q, new, masks, 0.18)


def test_two_streams():
    """Cut lengths on two streams at once, each with a workspace and outputs of its own."""
    import torch
    from paper_2109_08008_amd import nt
    cases = []
    for i, (new, lens) in enumerate((([5, 12], [3000, 1500]), ([17], [2800]))):
        pages = Pages(lens, 1, 64, 64, "f16", seed=i).fill(3)
        q = queries(17, 4, 64, "f16", seed=i, behind=0)
        masks = trees(new, i)
        want = run(pages, q, new, masks, 0.125, max_len=3000)
        check(want, pages, q, new, masks, 0.125)
        off = torch.tensor([sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32, device="cuda")
        mask = torch.tensor([w for m in masks for w in m], device="cuda")
        need = nt.nt_op_attn_tree_workspace(pages.cache, 4, len(new), 17, max(new), 3000)
        ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
        cases.append((pages, q, off, mask, len(new), max(new), need, ws, want, torch.full_like(want, 7.0),
                      torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(8):
        for pages, q, off, mask, n, most, need, ws, _, out, st in cases:
            nt.nt_op_attn_tree(pages.cache, q.data_ptr(), 256, 4, off.data_ptr(), mask.data_ptr(), pages.lens.data_ptr(), n,
                               17, most, 3000, 0.125, out.data_ptr(), 256, ws.data_ptr(), need, st.cuda_stream)
    torch.cuda.synchronize()
    for *_, want, out, _ in cases:
        assert torch.equal(out, want)


def test_pools_past_32_bits():
    """Pages whose distance from the pool's start passes 2^32 bytes."""
    import numpy as np
    import torch
    from paper_2109_08008_amd import nt
    small = Pages([300, 40], 4, 128, 256, "f16", seed=1).fill(2)
    n_pages = 18000
    k, v = (torch.empty(n_pages, 4, 256, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    table = np.full(small.table_np.shape, -1, np.int32)
    for b in range(2):
        for j in range(small.max_pages):
            pid = int(small.table_np[b, j])
            if pid >= 0:
                table[b, j] = n_pages - 1 - pid
                k[n_pages - 1 - pid], v[n_pages - 1 - pid] = small.k[pid], small.v[pid]
    d_table = torch.from_numpy(table).cuda()
    big = nt.kv_pages("f16", 4, 128, 256, n_pages, small.max_pages, k.data_ptr(), v.data_ptr(), d_table.data_ptr())
    q = queries(20, 8, 128, "f16")
    new = [12, 8]
    masks = trees(new, 1)
    want = run(small, q, new, masks, 0.09)
    old, small.cache = small.cache, big
    got = run(small, q, new, masks, 0.09)
    small.cache = old
    assert torch.equal(got, want)
    check(want, small, q, new, masks, 0.09)
