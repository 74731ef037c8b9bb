"""Attention of many query rows in float64, with the error its kernels may have, for the tests of
packed prompts and of new tokens over a paged cache."""
from tests.paged_util import EPS


def attention(q, k, v, seen, scale, dtype):
    """(out, bound) in float64 of q [rows, heads, dh] over k, v [keys, kv_heads, dh] (all float64, on one
    device): row i sees key j where seen[i, j]; what it does not see never counts, whatever it is.

    With u half a step of dtype, A = sum_j p_j |v_j| and o the output: the output's rounding u |o|; with
    16 bits each probability is off by at most u of itself, in the sum too, so that o is off by at most
    sum_j u p_j |v_j - o| <= u (A + |o|), and 1 + 4 u covers the second order; fp16 probabilities enter
    the product 2^7 times as large against a reference at most 2^8 below the row's largest, so that one
    below 2^-14 is off by 2^-25 of at least 2^7 at the largest: 2^-32 a key.  Scores are fp32 dot
    products of dh terms, scaled: off by at most (dh + 2) 2^-24 sum |q||k| |scale|; the exponential and
    its argument's rounding add 2^-20; each twice in p (its own and the sum's).  fp32 sums of n terms
    n 2^-24 A, and the factors of moved references and joins 2^-19 A."""
    import torch
    rows, heads, dh = q.shape
    group = heads // k.shape[1]
    u = EPS[dtype] / 2
    r = u if dtype != "f32" else 0.0
    out, bound = torch.zeros_like(q), torch.zeros_like(q)
    used = seen.any(0)
    zero = torch.zeros((), dtype=q.dtype, device=q.device)
    for h in range(heads):
        kk, vv = k[:, h // group], v[:, h // group]
        kk, vv = torch.where(used[:, None], kk, zero), torch.where(used[:, None], vv, zero)
        s = torch.where(seen, q[:, h] @ kk.t().contiguous() * scale, zero - float("inf"))
        m = s.amax(1, keepdim=True)
        e = torch.exp(s - torch.where(torch.isinf(m) & (m < 0), zero, m))
        z = e.sum(1, keepdim=True)
        p = e / torch.where(z == 0, zero + 1, z)
        o, a = p @ vv, p @ vv.abs()
        size = torch.where(seen, q[:, h].abs() @ kk.abs().t().contiguous(), zero).amax(1, keepdim=True) * abs(scale)
        ds = (dh + 2) * 2.0 ** -24 * size + 2.0 ** -20
        n = seen.sum(1, keepdim=True).double()
        err = u * o.abs() + r * (1 + 4 * u) * (a + o.abs()) + (2 * ds + n * 2.0 ** -24 + 2.0 ** -19) * a
        if dtype == "f16":      # (and the output's own subnormals)
            err = err + n * 2.0 ** -32 * (vv.abs().amax(0) + o.abs()) + 2.0 ** -25
        out[:, h], bound[:, h] = o, err
    return out, bound


def assert_rows(got, want, bound, what=""):
    """got is within bound of want where that is a number, and no number (or as infinite) where it is not."""
    import torch
    got = got.double()
    fine = torch.isfinite(want)
    assert bool(torch.isfinite(got[fine]).all()), what
    over = (got - want).abs() - bound
    assert float(over[fine].max()) <= 0 if bool(fine.any()) else True, (
        what, float(over[fine].max()), float((got - want).abs()[fine].max()))
    nan = torch.isnan(want)
    assert bool(torch.isnan(got[nan]).all()), what
    inf = torch.isinf(want)
    assert bool((got[inf] == want[inf]).all()), what
