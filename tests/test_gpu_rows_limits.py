"""GPU: attention of many query rows at the edges of what numbers hold, in each way that a row's keys are
shared out: over a tile's waves, over parts of a length, over neither."""
import pytest

from tests.paged_util import Pages, torch_dtype
from tests.test_gpu_prompt import check as check_prompt, make, run as run_prompt
from tests.test_gpu_tree import check as check_tree, queries, run as run_tree, trees

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
