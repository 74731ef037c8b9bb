"""Paged caches for the tests: pools whose unused cells hold NaN, scattered pages, and the
attention over them in float64, with the error its kernel may have."""
import numpy as np

EPS = {"f32": 2.0 ** -23, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}


def torch_dtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


class Pages:
    """Pools and table on the GPU for sequences of the given lengths; page ids are scattered, and
    every cell that no sequence holds is NaN."""

    def __init__(self, lens, kv_heads, d_head, page, dtype="f16", fp8=False, seed=0, spare=2, extra_pages=0, device="cuda"):
        import torch
        from paper_2109_08008_amd import nt
        rng = np.random.default_rng(seed)
        self.lens_list, self.kv_heads, self.d_head, self.page = list(lens), kv_heads, d_head, page
        self.dtype, self.fp8 = dtype, fp8
        need = [(n + page - 1) // page for n in lens]
        self.max_pages = max([1] + need) + extra_pages
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        self.table_np = np.full((len(lens), self.max_pages), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table_np[b, :n] = order[at:at + n]
            at += n
        shape = (self.n_pages, kv_heads, page, d_head)
        if fp8:
            self.k, self.v = (torch.full(shape, 0x7F, dtype=torch.uint8, device=device) for _ in range(2))
        else:
            self.k, self.v = (torch.full(shape, float("nan"), dtype=torch_dtype(dtype), device=device) for _ in range(2))
        self.table = torch.from_numpy(self.table_np).to(device)
        self.lens = torch.tensor(list(lens), dtype=torch.int32, device=device)
        self.cache = nt.kv_pages(dtype, kv_heads, d_head, page, self.n_pages, self.max_pages, self.k.data_ptr(),
                                 self.v.data_ptr(), self.table.data_ptr(), fp8=fp8)

    def retable(self, table_np):
        import torch
        self.table_np = table_np
        self.table.copy_(torch.from_numpy(table_np))

    def fill(self, seed, scale=1.0):
        """Random keys and values at every held position (exact in the cache's type)."""
        import torch
        g = torch.Generator().manual_seed(seed)
        for pool in (self.k, self.v):
            for b, n in enumerate(self.lens_list):
                for j in range((n + self.page - 1) // self.page):
                    rows = min(self.page, n - j * self.page)
                    x = torch.randn(self.kv_heads, rows, self.d_head, generator=g) * scale
                    x = x.to(torch.float8_e4m3fn).view(torch.uint8) if self.fp8 else x.to(torch_dtype(self.dtype))
                    pid = int(self.table_np[b, j])
                    if 0 <= pid < self.n_pages:
                        pool[pid, :, :rows] = x.to(pool.device)
        return self

    def values(self, pool):
        """The pool in float64 on the host."""
        import torch
        x = pool.view(torch.float8_e4m3fn) if self.fp8 else pool
        return x.cpu().to(torch.float64)

    def attention(self, q, scale, lens=None):
        """(out, bound) in float64: softmax attention of q [n, heads, d_head] over the held
        positions, and what the kernel's roundings may add up to.

        With u half a step of dtype, A = sum_j p_j |V_j|: the output's rounding u |o|, the
        probabilities' u A (fp16: and 2^-25 a probability below its normal range, against the
        largest, which is 1 of a sum of at least 1); scores are fp32 dot products of d_head
        terms, scaled: off by at most (d_head + 2) 2^-24 sum |q||K| scale, and the exponential
        adds 2^-21, each twice in p (its own and the sum's); fp32 sums of n terms n 2^-24 A,
        and a join's factors 2^-20 A."""
        import torch
        k, v = self.values(self.k), self.values(self.v)
        heads = q.shape[1]
        group = heads // self.kv_heads
        out = torch.zeros(q.shape, dtype=torch.float64)
        bound = torch.zeros(q.shape, dtype=torch.float64)
        u = EPS[self.dtype] / 2
        for b in range(q.shape[0]):
            n = min((self.lens_list if lens is None else lens)[b], self.max_pages * self.page)
            pos = [p for p in range(max(n, 0)) if 0 <= self.table_np[b, p // self.page] < self.n_pages]
            if not pos:
                continue
            pid = torch.tensor([int(self.table_np[b, p // self.page]) for p in pos])
            slot = torch.tensor([p % self.page for p in pos])
            for h in range(heads):
                kk, vv = k[pid, h // group, slot], v[pid, h // group, slot]
                qq = q[b, h].cpu().to(torch.float64)
                p = torch.softmax(kk @ qq * scale, 0)
                o, a = p @ vv, p @ vv.abs()
                ds = (self.d_head + 2) * 2.0 ** -24 * float((kk.abs() @ qq.abs()).max()) * abs(scale) + 2.0 ** -21
                out[b, h] = o
                bound[b, h] = u * o.abs() + (u if self.dtype != "f32" else 0.0) * a + 2 * ds * a + (
                    len(pos) * 2.0 ** -24 + 2.0 ** -20) * a
                if self.dtype == "f16":
                    bound[b, h] += len(pos) * 2.0 ** -25 * vv.abs().amax(0) + 2.0 ** -25
        return out, bound


def attend(pages, q, scale, max_len=None, n_seqs=None, lens=None, out=None, ws=None, stream=None):
    """nt_op_attn_paged on q [rows, heads, d_head] (rows may be strided); returns out."""
    import torch
    from paper_2109_08008_amd import nt
    n = len(pages.lens_list) if n_seqs is None else n_seqs
    heads = q.shape[1]
    max_len = max([0] + pages.lens_list) if max_len is None else max_len
    if out is None:
        out = torch.full((q.shape[0], heads, pages.d_head), 7.0, dtype=q.dtype, device=q.device)
    need = nt.nt_op_attn_paged_workspace(pages.cache, heads, n, max_len)
    if ws is None:
        ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device=q.device)   # NaN in every float
    nt.nt_op_attn_paged(pages.cache, q.data_ptr(), q.stride(0), heads, (pages.lens if lens is None else lens).data_ptr(), n,
                        max_len, scale, out.data_ptr(), out.stride(0), ws.data_ptr() if need else None, need, stream)
    return out


def assert_within(got, want, bound, what=""):
    import torch
    got = got.cpu().to(torch.float64)
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - bound
    assert float(over.max()) <= 0, (what, float(over.max()), float((got - want).abs().max()))


def attention_of_many(pages, q, scale, p_rel, p_abs):
    """attention() of many sequences at once, in float64 on the GPU, with the probabilities' part of the
    bound as given: each is off by at most p_rel of itself and p_abs of the largest."""
    import torch
    n, heads, dh = q.shape
    hkv, group, page = pages.kv_heads, heads // pages.kv_heads, pages.page
    length = pages.max_pages * page
    out = torch.empty(q.shape, dtype=torch.float64)
    bound = torch.empty(q.shape, dtype=torch.float64)
    u = EPS[pages.dtype] / 2
    step = max(1, (1 << 25) // (hkv * length * dh))
    lens = torch.tensor(pages.lens_list, device=q.device)
    for b in range(0, n, step):
        table = pages.table[b:b + step].long()
        real = (table >= 0) & (table < pages.n_pages)
        held = real.repeat_interleave(page, 1) & (torch.arange(length, device=q.device) < lens[b:b + step, None])

        def cells(pool):   # [n, hkv, length, dh], 0 where nothing is held
            x = pool[torch.where(real, table, torch.zeros_like(table))]
            x = (x.view(torch.float8_e4m3fn).float() if pages.fp8 else x).double()
            x = x.permute(0, 2, 1, 3, 4).reshape(-1, hkv, length, dh)
            return torch.where(held[:, None, :, None], x, torch.zeros_like(x)).contiguous()

        k, v = cells(pages.k), cells(pages.v)
        qq = q[b:b + step].double().reshape(-1, hkv, group, dh).transpose(2, 3).contiguous()
        s = torch.matmul(k, qq).transpose(2, 3).contiguous() * scale                      # [n, hkv, group, length]
        size = torch.matmul(k.abs(), qq.abs()).amax(2)[..., None] * abs(scale)
        s = s.masked_fill(~held[:, None, None], -float("inf"))
        m = s.amax(3, keepdim=True)
        e = torch.exp(s - torch.where(torch.isfinite(m), m, torch.zeros_like(m)))
        z = e.sum(3, keepdim=True)
        p = e / torch.where(z == 0, torch.ones_like(z), z)
        o, a = torch.matmul(p, v), torch.matmul(p, v.abs())
        ds = (dh + 2) * 2.0 ** -24 * size + 2.0 ** -21
        keys = held.sum(1).double()[:, None, None, None]
        err = u * o.abs() + p_rel * a + p_abs * keys * v.abs().amax(2)[:, :, None] + (2 * ds + keys * 2.0 ** -24 + 2.0 ** -20) * a
        if pages.dtype == "f16":
            err = err + 2.0 ** -25
        out[b:b + step] = o.reshape(-1, heads, dh).cpu()
        bound[b:b + step] = err.reshape(-1, heads, dh).cpu()
    return out, bound
