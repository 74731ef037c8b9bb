"""GPU: attention of many query rows at the edges of what numbers hold, in each way that a row's keys are
shared out: over a tile's waves, over parts of a length, over neither."""
import pytest

from tests.paged_util import Pages, torch_dtype
from tests.rows_util import assert_rows, attention
from tests.test_gpu_prompt import check as check_prompt, make, run as run_prompt, split
from tests.test_gpu_tree import cells, check as check_tree, queries, run as run_tree, trees

pytestmark = pytest.mark.gpu

# lengths of prompts and heads, so that tiles of 16 (four waves and two), 32, 64 and 128 rows and those of
# short sequences are taken
PROMPTS = [(2, [300, 5]), (24, [40, 1, 17, 33, 16, 15, 65, 2]), (40, [200, 31, 99]), (64, [300, 200, 65]),
           (96, [700, 324]), (96, [33, 16, 140, 64, 17, 63, 65, 2] * 3)]
PROMPT_IDS = ["16", "pair", "32", "64", "128", "short"]


def large_values(shape, dtype, size, seed):
    """Values of both signs, of size .. size / 2."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = size * (1 - 0.5 * torch.rand(shape, generator=g, dtype=torch.float64))
    x *= torch.where(torch.rand(shape, generator=g) < 0.5, -1.0, 1.0)
    return x.to(torch_dtype(dtype)).cuda()


# ---- averages of values whose sums pass fp32's largest number -----------------------------
# The largest number of fp32 is 3.4e38; 3e38 is an eighth below it, so that the errors that `attention` allows
# do not carry an average past it.
@pytest.mark.parametrize("dtype,size", [("bf16", 3e38), ("f32", 3e38), ("bf16", 1e36), ("f32", 1e36), ("f16", 65504.0)])
@pytest.mark.parametrize("same_sign", [True, False])
@pytest.mark.parametrize("heads,lens", PROMPTS, ids=PROMPT_IDS)
def test_large_values_of_prompts(heads, lens, same_sign, dtype, size):
    """Finite values have a finite average, however many keys share the weight."""
    dh, hkv = 128 if heads == 24 else 64, heads // 8 or 1
    heads = hkv * 8 if heads > 8 else heads
    x, off, rows = make(lens, heads, hkv, dh, dtype, seed=heads, scale=0.1)
    v = large_values((rows, hkv * dh), dtype, size, heads)
    x[:, (heads + hkv) * dh:] = v.abs() if same_sign else v
    for causal in (True, False):
        got = run_prompt(x, off, rows, heads, hkv, dh, dtype, causal, 0.1)
        check_prompt(got, x, off, heads, hkv, dh, dtype, causal, 0.1)


@pytest.mark.parametrize("dtype,size", [("bf16", 3e38), ("f32", 3e38), ("bf16", 1e35), ("f32", 1e35)])
def test_many_equal_scores(dtype, size):
    """4096 equal scores: their sum passes the largest number from 2^12 below it on."""
    import torch
    n, dh = 4096, 64
    x, off, rows = make([n], 1, 1, dh, dtype, seed=5)
    x[:, :2 * dh] = 0
    x[:, 2 * dh:] = large_values((n, dh), dtype, size, 3).abs()
    check_prompt(run_prompt(x, off, rows, 1, 1, dh, dtype, True, 1.0), x, off, 1, 1, dh, dtype, True, 1.0)
    # values all alike: their average is within the roundings of themselves
    x[:, 2 * dh:] = torch.tensor(size, dtype=x.dtype)
    check_prompt(run_prompt(x, off, rows, 1, 1, dh, dtype, True, 1.0), x, off, 1, 1, dh, dtype, True, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group,new", [(1, 3), (4, 4), (4, 16), (4, 40)])
@pytest.mark.parametrize("lens", [(100, 250), (5003, 700), (30000, 40)], ids=str)
@pytest.mark.parametrize("size", [3e38, 1e36])
def test_large_values_over_a_cache(size, lens, group, new, dtype):
    """The same over a cache, where waves and parts of a length are joined."""
    news = [new, new]
    pages = Pages(list(lens), 1, 64, 64, dtype, seed=6).fill(7)
    pages.v.copy_(large_values(tuple(pages.v.shape), dtype, size, 8))
    q = queries(2 * new, group, 64, dtype) * 0.1
    for masks in (trees(news, 2), None):
        check_tree(run_tree(pages, q, news, masks, 0.125, n_rows=2 * new), pages, q, news, masks, 0.125)
    pages.v.abs_()
    check_tree(run_tree(pages, q, news, None, 0.125, n_rows=2 * new), pages, q, news, None, 0.125)


# ---- scores of -inf -------------------------------------------------------------------
# A softmax over scores of -inf alone is no number; beside one finite score they weigh nothing.
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("heads,lens", PROMPTS, ids=PROMPT_IDS)
def test_nothing_but_scores_of_minus_infinity(heads, lens, dtype, causal):
    """Every second sequence has keys of -inf: all of them, or (the third, seventh ..) all but the last."""
    import torch
    dh, hkv = 128 if heads == 24 else 64, heads // 8 or 1
    heads = hkv * 8 if heads > 8 else heads
    x, off, rows = make(lens, heads, hkv, dh, dtype, seed=heads)
    x[:, :heads * dh:dh] = x[:, :heads * dh:dh].abs() + 0.5          # channel 0 of every query is positive
    for b in range(0, len(lens), 2):
        end = off[b + 1] - (1 if b % 4 == 2 else 0)
        x[off[b]:end, heads * dh:(heads + hkv) * dh:dh] = float("-inf")
    got = run_prompt(x, off, rows, heads, hkv, dh, dtype, causal, 0.1)
    q, k, v = split(torch.where(torch.isinf(x), torch.zeros_like(x), x), heads, hkv, dh)
    for b, n in enumerate(lens):
        lo, hi = off[b], off[b + 1]
        seen = torch.ones(n, n, dtype=torch.bool, device="cuda")
        seen = seen.tril() if causal else seen
        if b % 2 == 0:
            seen[:, :n - (1 if b % 4 == 2 else 0)] = False
        want, bound = attention(q[lo:hi], k[lo:hi], v[lo:hi], seen, 0.1, dtype)
        some = seen.any(1)
        mine = got[lo:hi].reshape(n, heads, dh)
        assert bool(torch.isnan(mine[~some]).all()), (b, n)
        if bool(some.any()):
            assert_rows(mine[some], want[some], bound[some], (b, n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_overflow_downwards(dtype):
    """Finite queries and keys whose product is below fp32's range: no number, as above it."""
    import torch
    lens, dh = [20, 70], 64
    for sign in (1, -1):
        x, off, rows = make(lens, 1, 1, dh, dtype, seed=2)
        x[:20, :dh] = 1e25
        x[:20, dh:2 * dh] = sign * 1e25
        got = run_prompt(x, off, rows, 1, 1, dh, dtype, True, 0.1)
        assert bool(torch.isnan(got[:20]).all())
        q, k, v = split(x[20:], 1, 1, dh)
        seen = torch.ones(70, 70, dtype=torch.bool, device="cuda").tril()
        want, bound = attention(q, k, v, seen, 0.1, dtype)
        assert_rows(got[20:].reshape(70, 1, dh), want, bound)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("group,new", [(1, 3), (4, 4), (4, 16), (4, 40)])
@pytest.mark.parametrize("length", [50, 250, 5003])
@pytest.mark.parametrize("tree", [True, False])
def test_scores_of_minus_infinity_over_a_cache(tree, length, group, new, dtype):
    """Keys of -inf in the whole context, in most of it (parts that hold nothing else), and in new tokens."""
    import torch
    base = length - new
    masks = [[1 << i for i in range(new)]] if tree else None        # tokens that see the context and themselves
    q = queries(new, group, 64, dtype, behind=0)
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    for finite in ([], [0], [base - 1], [base + 1], [base // 2, base]):
        pages = Pages([length], 1, 64, 16, dtype, seed=3).fill(4)
        clean = pages.k.clone()
        for p in range(length):
            if p not in finite:
                pages.k[int(pages.table_np[0, p // 16]), 0, p % 16, 0] = float("-inf")
        got = run_tree(pages, q, [new], masks, 0.125)
        pages.k.copy_(clean)
        k, _ = cells(pages, pages.k, 0, length)
        v, _ = cells(pages, pages.v, 0, length)
        seen = torch.zeros(new, length, dtype=torch.bool, device="cuda")
        for p in finite:
            for i in range(new):
                seen[i, p] = p < base or (p - base == i if tree else p - base <= i)
        want, bound = attention(q.double(), k, v, seen, 0.125, dtype)
        some = seen.any(1)
        assert bool(torch.isnan(got[~some]).all()), finite
        if bool(some.any()):
            assert_rows(got[some], want[some], bound[some], finite)


@pytest.mark.parametrize("length", [6, 100, 3000])
def test_holes_and_empty_masks_beside_minus_infinity(length):
    """Rows without a key that they see are zero, whatever stands in holes and in keys that others see."""
    import torch
    new = 6
    pages = Pages([length, length], 1, 64, 16, "f16", seed=3).fill(4)
    pages.k[:, :, :, 0] = float("-inf")
    table = pages.table_np.copy()
    table[0, :] = -1                                 # the first sequence has no page
    pages.retable(table)
    q = queries(2 * new, 4, 64, "f16")
    q[:, :, 0] = 1.0
    for masks in ([[0] * new, [0] * new], None):
        got = run_tree(pages, q, [new, new], masks, 0.125)
        assert bool((got[:new] == 0).all())
        if masks is not None and length == new:
            assert bool((got[new:2 * new] == 0).all())
        else:
            assert bool(torch.isnan(got[new:2 * new]).all())


# ---- a scale of 0 -----------------------------------------------------------------------
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-40, -1e-40])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
def test_queries_that_are_no_numbers_at_scale_0(bad, dtype, scale):
    """0 times what is no number is none, whether or not another row of the wave is formed again; the others
    are means of their values."""
    import torch
    lens, h, hkv, dh = [40, 100], 2, 1, 64
    for broken_value in (False, True):
        x, off, rows = make(lens, h, hkv, dh, dtype, seed=4)
        x[17, 3] = float(bad)                        # head 0 of a row of either sequence
        x[60, dh + 5] = float(bad)                   # head 1
        if broken_value:
            x[39, (h + hkv) * dh:] = float("nan")    # seen by the first one's last row alone
        got = run_prompt(x, off, rows, h, hkv, dh, dtype, True, scale).reshape(rows, h, dh)
        hit = torch.zeros(rows, h, dtype=torch.bool, device="cuda")
        hit[17, 0] = hit[60, 1] = True
        hit[39] = broken_value
        assert bool(torch.isnan(got[hit]).all())
        q, k, v = split(torch.nan_to_num(x, posinf=0.0, neginf=0.0), h, hkv, dh)
        for b, n in enumerate(lens):
            lo, hi = off[b], off[b + 1]
            seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
            want, bound = attention(q[lo:hi], k[lo:hi], v[lo:hi], seen, 0.0, dtype)
            ok = ~hit[lo:hi]
            assert_rows(got[lo:hi][ok], want[ok], bound[ok], (b, broken_value))


@pytest.mark.parametrize("dtype,fp8", [("f16", False), ("f16", True), ("bf16", False), ("f32", False)])
def test_scale_0_over_a_cache(dtype, fp8):
    """The same for new tokens over a cache, alone and in a tree."""
    import torch
    new = [3, 20]
    pages = Pages([60, 700], 1, 64, 16, dtype, fp8, seed=2).fill(3)
    q = queries(23, 4, 64, dtype, behind=0)
    q[1, 2, 7] = float("nan")
    q[9, 0, 0] = float("inf")
    hit = torch.isnan(q).any(2) | torch.isinf(q).any(2)
    clean = torch.nan_to_num(q, posinf=0.0)
    for masks in (trees(new, 4), None):
        got = run_tree(pages, q, new, masks, 0.0)
        assert bool(torch.isnan(got[hit]).all())
        want = run_tree(pages, clean, new, masks, 0.0)
        check_tree(want, pages, clean, new, masks, 0.0)
        got[hit] = want[hit]
        check_tree(got, pages, clean, new, masks, 0.0)
