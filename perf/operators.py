"""The operators of an incremental decoder over a paged key/value cache, as timed and compared cases.

Four kinds of case, each one call of an entry point of ``paper_2109_08008_amd.nt``:

* ``append``  new tokens' keys and values into a paged cache, ``nt_op_kv_append``;
* ``attn``    attention of one new token a sequence over such a cache, ``nt_op_attn_paged``;
* ``gated``   the input half of a gated feed-forward block, ``nt_op_gemm_gated``;
* ``logp``    log-probabilities of given tokens with log-sum-exp, entropy and the best
              alternatives of each row of logits, ``nt_op_token_logp``.

``run`` computes them in elementary torch operations (``own`` false) or through the library.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
ACTS = ("silu", "gelu", "gelu_tanh", "relu")
LN_EPS = 1e-5
NONE = 2 ** 31 - 1      # index of an alternative that a row does not have
MAX_CACHE = 1 << 29     # n_seqs * longest * kv_heads * d_head of a drawn cache
MAX_FLOPS = 4 * 16384 * 4096 * 1024
MAX_LOGITS = 8192 * 32001


def listed():
    return [
        # one step of 96 live hypotheses of a base model: one new key and value each
        {"name": "append_step", "kind": "append", "dtype": "f16", "fp8": False, "n_seqs": 96, "kv_heads": 8,
         "d_head": 64, "page": 16, "new_min": 1, "new_max": 1, "longest": 160},
        # prompts (or forced prefixes) of 256 requests enter an FP8 cache at once, ragged
        {"name": "append_prompts_fp8", "kind": "append", "dtype": "f16", "fp8": True, "n_seqs": 256, "kv_heads": 16,
         "d_head": 64, "page": 32, "new_min": 1, "new_max": 150, "longest": 300},
        # a decoder step of 64 sentences of ordinary length: few keys, latency counts
        {"name": "attn_sentences", "kind": "attn", "dtype": "f16", "fp8": False, "n_seqs": 64, "heads": 8, "kv_heads": 8,
         "d_head": 64, "page": 16, "shortest": 1, "longest": 48},
        # a wide decoder at an ordinary batch (540 x beam 4) with targets of a few hundred tokens, bf16
        {"name": "attn_batch_bf16", "kind": "attn", "dtype": "bf16", "fp8": False, "n_seqs": 2160, "heads": 16,
         "kv_heads": 16, "d_head": 64, "page": 32, "shortest": 1, "longest": 231},
        # whole documents, ragged, four query heads to a key head
        {"name": "attn_documents", "kind": "attn", "dtype": "f16", "fp8": False, "n_seqs": 16, "heads": 32, "kv_heads": 8,
         "d_head": 128, "page": 64, "shortest": 2048, "longest": 32768},
        # one request with a very long FP8 cache: only the split over its length fills the GPU
        {"name": "attn_one_long_fp8", "kind": "attn", "dtype": "f16", "fp8": True, "n_seqs": 1, "heads": 16, "kv_heads": 4,
         "d_head": 128, "page": 128, "shortest": 131001, "longest": 131001},
        # a step of three live rows: the weights are all there is to read
        {"name": "gated_tokens", "kind": "gated", "dtype": "f16", "m": 3, "n": 2048, "k": 512, "act": "silu", "ln": True,
         "bias": True},
        # a wide decoder's step at an ordinary batch, its pre-norm LayerNorm folded in
        {"name": "gated_step_ln", "kind": "gated", "dtype": "f16", "m": 2160, "n": 4096, "k": 1024, "act": "silu",
         "ln": True, "bias": True},
        # a wide encoder's full batch of 16384 tokens in bf16, no bias
        {"name": "gated_enc_bf16", "kind": "gated", "dtype": "bf16", "m": 16384, "n": 4096, "k": 1024,
         "act": "gelu_tanh", "ln": False, "bias": False},
        # the answer's first token of two requests over a large vocabulary
        {"name": "logp_two_rows", "kind": "logp", "dtype": "f32", "rows": 2, "vocab": 131072, "k": 20, "n_tok": 1,
         "masked": 0.0},
        # a step's fp32 logits (325 x beam 4) with the forbidden words at -inf
        {"name": "logp_step", "kind": "logp", "dtype": "f32", "rows": 1300, "vocab": 32000, "k": 8, "n_tok": 1,
         "masked": 0.05},
        # every position of a forced batch, 16-bit logits whose rows start at any alignment
        {"name": "logp_forced_bf16", "kind": "logp", "dtype": "bf16", "rows": 8192, "vocab": 32001, "k": 5, "n_tok": 2,
         "masked": 0.0},
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("append", "attn", "attn", "gated", "gated", "logp"))
    dtype = rng.choice(("f16", "f16", "bf16", "bf16", "f32"))
    if kind in ("append", "attn"):
        fp8 = dtype == "f16" and rng.random() < 0.4
        c = {"kind": kind, "dtype": dtype, "fp8": fp8, "kv_heads": rng.choice((1, 2, 3, 4, 8, 16)),
             "d_head": rng.choice((32, 64, 128)), "page": rng.choice((16, 32, 64, 128, 256))}
        width = c["kv_heads"] * c["d_head"]
        if kind == "append":
            c["n_seqs"] = spread(1, 1024)
            c["new_min"] = 1
            c["new_max"] = 1 if rng.random() < 0.5 else spread(2, max(2, min(2000, (1 << 25) // (width * c["n_seqs"]))))
            c["longest"] = c["new_max"] + spread(1, 2000)
            while c["n_seqs"] * (c["longest"] + c["page"]) * width > MAX_CACHE // 4:
                c["n_seqs"] = (c["n_seqs"] + 1) // 2
            return c
        c["heads"] = c["kv_heads"] * rng.choice((1, 1, 2, 3, 4, 8, 20))
        c["n_seqs"] = spread(1, 2048)
        c["longest"] = spread(1, 120000)
        while c["n_seqs"] * (c["longest"] + c["page"]) * width > MAX_CACHE:
            c["n_seqs"], c["longest"] = (c["n_seqs"] + 1) // 2, max(1, c["longest"] * 3 // 4)
        c["shortest"] = max(1, int(c["longest"] * rng.choice((0.01, 0.3, 1.0))))
        return c
    if kind == "gated":
        k = rng.choice((64, 128, 256, 320, 512, 576, 768, 1024))
        n = rng.choice((2 * k, 4 * k, 8 * k // 3, spread(16, 4096)))
        m = spread(1, 16384)
        if dtype == "f32":
            m = min(m, 4096)
        while 4 * m * n * k > MAX_FLOPS:
            m = (m + 1) // 2
        return {"kind": kind, "dtype": dtype, "m": m, "n": n, "k": k, "act": rng.choice(ACTS), "ln": rng.random() < 0.4,
                "bias": rng.random() < 0.6}
    vocab = spread(1000, 150000)
    rows = spread(1, 8192)
    while rows * vocab > MAX_LOGITS // (2 if dtype == "f32" else 1):
        rows = (rows + 1) // 2
    return {"kind": kind, "dtype": dtype, "rows": rows, "vocab": vocab, "k": rng.choice((0, 1, 4, 5, 8, 20, 32)),
            "n_tok": rng.choice((1, 1, 1, 2, 7)), "masked": rng.choice((0.0, 0.0, 0.1))}


def _lengths(case):
    """The sequences' lengths (new ones included) and new rows: the case's own, whatever the seed."""
    r = random.Random("%(kind)s %(n_seqs)d %(longest)d %(page)d" % case)
    if case["kind"] == "attn":
        lens = [r.randint(case["shortest"], case["longest"]) for _ in range(case["n_seqs"])]
        if case["n_seqs"] > 8:
            lens[r.randrange(case["n_seqs"])] = 0       # a slot that no request holds at the moment
        return lens, [1] * case["n_seqs"]
    new = [r.randint(case["new_min"], case["new_max"]) for _ in range(case["n_seqs"])]
    return [r.randint(n, case["longest"]) for n in new], new


def _cell(case):
    return 1 if case.get("fp8") else BYTES[case["dtype"]]


def work(case):
    """Bytes and operations that one pass cannot do without: inputs read once, outputs written once."""
    eb = BYTES[case["dtype"]]
    if case["kind"] == "append":
        n = sum(_lengths(case)[1]) * 2 * case["kv_heads"] * case["d_head"]
        return {"bytes": float(n * (eb + _cell(case))), "flops": 0.0}
    if case["kind"] == "attn":
        keys = sum(_lengths(case)[0])
        return {"bytes": float(keys * 2 * case["kv_heads"] * case["d_head"] * _cell(case)
                               + 2 * case["n_seqs"] * case["heads"] * case["d_head"] * eb),
                "flops": 4.0 * keys * case["heads"] * case["d_head"]}
    if case["kind"] == "gated":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": float((m * k + 2 * n * k + m * n) * eb), "flops": 4.0 * m * n * k}
    r, v = case["rows"], case["vocab"]
    return {"bytes": float(r * v * eb + r * (2 * case["n_tok"] + 2 + 2 * case["k"]) * 4), "flops": 5.0 * r * v}


def _normal(gen, *shape, scale=1.0, shift=0.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    dt = TORCH[case["dtype"]]
    if case["kind"] in ("append", "attn"):
        lens, new = _lengths(case)
        hkv, dh, page, n = case["kv_heads"], case["d_head"], case["page"], case["n_seqs"]
        need = [(x + page - 1) // page for x in lens]
        most = max(1, max(need))
        n_pages = sum(need) + 3
        r = random.Random(seed)
        order = list(range(n_pages))      # a pool in use for a while: pages lie anywhere
        r.shuffle(order)
        table = torch.full((n, most), -1, dtype=torch.int32)
        at = 0
        for b, p in enumerate(need):
            table[b, :p] = torch.tensor(order[at:at + p], dtype=torch.int32)
            at += p
        cell = torch.float8_e4m3fn if case["fp8"] else dt
        s["table"] = table.cuda()
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["max_len"] = max(lens)
        if case["kind"] == "append":
            off = [0]
            for x in new:
                off.append(off[-1] + x)
            s["off"] = None if max(new) == 1 else torch.tensor(off, dtype=torch.int32, device="cuda")
            s["rows"] = off[-1]
            # the projection's rows hold query, key and value side by side
            s["qkv"] = _normal(gen, off[-1], 3 * hkv * dh, dtype=dt)
            s["k"] = torch.zeros(n_pages, hkv, page, dh, dtype=torch.uint8 if case["fp8"] else dt, device="cuda").view(cell)
            s["v"] = torch.zeros(n_pages, hkv, page, dh, dtype=torch.uint8 if case["fp8"] else dt, device="cuda").view(cell)
        else:
            s["q"] = _normal(gen, n, case["heads"], dh, dtype=dt)
            s["k"] = torch.empty(n_pages, hkv, page, dh, dtype=cell, device="cuda")
            s["v"] = torch.empty(n_pages, hkv, page, dh, dtype=cell, device="cuda")
            for p in range(0, n_pages, 4096):
                cut = s["k"][p:p + 4096].shape
                s["k"][p:p + 4096] = _normal(gen, *cut).to(cell)
                s["v"][p:p + 4096] = _normal(gen, *cut, shift=0.1).to(cell)
            s["out"] = torch.empty(n, case["heads"], dh, dtype=dt, device="cuda")
            s["scale"] = dh ** -0.5
        if own:
            from paper_2109_08008_amd import nt
            s["cache"] = nt.kv_pages(case["dtype"], hkv, dh, page, n_pages, most, s["k"].data_ptr(), s["v"].data_ptr(),
                                     s["table"].data_ptr(), fp8=case["fp8"])
            if case["kind"] == "attn":
                need = nt.nt_op_attn_paged_workspace(s["cache"], case["heads"], n, s["max_len"])
                s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    elif case["kind"] == "gated":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"] = _normal(gen, m, k, scale=1.5 if case["ln"] else 1.0, shift=0.2 if case["ln"] else 0.0, dtype=dt)
        s["bt"] = _normal(gen, 2 * n, k, scale=k ** -0.5, dtype=dt)      # gate rows, then up rows
        s["bias"] = _normal(gen, 2 * n, scale=0.3) if case["bias"] else None
        s["colsum"] = s["bt"].float().sum(1) if case["ln"] else None
        s["out"] = torch.empty(m, n, dtype=dt, device="cuda")
    else:
        r, v, k = case["rows"], case["vocab"], case["k"]
        s["tokens"] = torch.randint(0, v, (r, case["n_tok"]), generator=gen, device="cuda", dtype=torch.int32)
        x = torch.empty(r, v, dtype=dt, device="cuda")
        for i in range(0, r, 512):
            cut = _normal(gen, min(512, r - i), v, scale=3.0)
            if case["masked"]:      # forbidden words, none of them a given token
                out = torch.rand(cut.shape, generator=gen, device="cuda") < case["masked"]
                cut[out.scatter_(1, s["tokens"][i:i + 512].long(), False)] = -math.inf
            x[i:i + 512] = cut.to(dt)
        s["logits"] = x
        s["logp"] = torch.empty(r, case["n_tok"], device="cuda")
        s["lse"] = torch.empty(r, device="cuda")
        s["entropy"] = torch.empty(r, device="cuda")
        s["topi"] = torch.empty(r, k, dtype=torch.int32, device="cuda")
        s["toplp"] = torch.empty(r, k, device="cuda")
        if own:
            from paper_2109_08008_amd import nt
            need = nt.nt_op_token_logp_workspace(case["dtype"], r, v, k)
            s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return s


def _run_own(s):
    from paper_2109_08008_amd import nt
    c = s["case"]
    if c["kind"] == "append":
        w, eb = c["kv_heads"] * c["d_head"], BYTES[c["dtype"]]
        base = s["qkv"].data_ptr()
        nt.nt_op_kv_append(s["cache"], base + w * eb, base + 2 * w * eb, 3 * w,
                           s["off"].data_ptr() if s["off"] is not None else None, s["lens"].data_ptr(), c["n_seqs"],
                           s["rows"])
        return {"k": s["k"], "v": s["v"]}
    if c["kind"] == "attn":
        w = c["heads"] * c["d_head"]
        nt.nt_op_attn_paged(s["cache"], s["q"].data_ptr(), w, c["heads"], s["lens"].data_ptr(), c["n_seqs"], s["max_len"],
                            s["scale"], s["out"].data_ptr(), w, s["ws"].data_ptr(), s["ws"].numel())
        return s["out"]
    if c["kind"] == "gated":
        nt.nt_op_gemm_gated(c["dtype"], s["a"].data_ptr(), c["k"], s["bt"].data_ptr(), c["m"], c["n"], c["k"], c["act"],
                            s["bias"].data_ptr() if c["bias"] else None, s["out"].data_ptr(), c["n"],
                            d_colsum=s["colsum"].data_ptr() if c["ln"] else None, ln_eps=LN_EPS)
        return s["out"]
    nt.nt_op_token_logp(c["dtype"], s["logits"].data_ptr(), c["vocab"], c["rows"], c["vocab"], s["tokens"].data_ptr(),
                        c["n_tok"], c["k"], s["logp"].data_ptr(), s["lse"].data_ptr(), s["entropy"].data_ptr(),
                        s["topi"].data_ptr() if c["k"] else None, s["toplp"].data_ptr() if c["k"] else None,
                        s["ws"].data_ptr(), s["ws"].numel())
    return {n: s[n] for n in ("logp", "lse", "entropy") + (("topi", "toplp") if c["k"] else ())}


# ---- plain forms -------------------------------------------------------------------------
def _append(s, c):
    w, page, n = c["kv_heads"] * c["d_head"], c["page"], c["n_seqs"]
    rows = torch.arange(s["rows"], device="cuda")
    if s["off"] is None:
        seq, pos = rows, s["lens"].long() - 1
    else:
        off = s["off"].long()
        seq = torch.searchsorted(off[1:], rows, right=True)
        pos = s["lens"].long()[seq] - (off[seq + 1] - rows)
    pages = s["table"][seq, pos // page].long()
    for name, at in (("k", w), ("v", 2 * w)):
        x = s["qkv"][:, at:at + w].reshape(-1, c["kv_heads"], c["d_head"])
        pool = s[name]
        if c["fp8"]:
            x = x.float().clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
            pool = pool.view(torch.uint8)
        pool[pages, :, pos % page] = x
    return {"k": s["k"], "v": s["v"]}


def _attn(s, c):
    n, h, hkv, dh = c["n_seqs"], c["heads"], c["kv_heads"], c["d_head"]
    at = s["table"].long().clamp(min=0)
    length = at.shape[1] * c["page"]

    def keys(pool):     # [n, hkv, length, dh]
        if c["fp8"]:
            x = pool.view(torch.uint8)[at].view(torch.float8_e4m3fn).float()
        else:
            x = pool[at].float()
        return x.permute(0, 2, 1, 3, 4).reshape(n, hkv, length, dh)

    q = (s["q"].float() * s["scale"]).reshape(n, hkv, h // hkv, dh).transpose(2, 3).contiguous()
    x = torch.matmul(keys(s["k"]), q)      # [n, hkv, length, group]
    beyond = torch.arange(length, device="cuda")[None, :] >= s["lens"][:, None]
    x = x.masked_fill(beyond[:, None, :, None], -math.inf)
    m = x.amax(2, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
    z = e.sum(2, keepdim=True)
    p = (e / torch.where(z == 0, torch.ones_like(z), z)).transpose(2, 3).contiguous()
    return torch.matmul(p, keys(s["v"])).reshape(n, h, dh).to(TORCH[c["dtype"]])


def _act(g, name):
    if name == "relu":
        return torch.clamp(g, min=0.0)
    if name == "silu":
        return g / (1.0 + torch.exp(-g))
    if name == "gelu":
        return 0.5 * g * (1.0 + torch.erf(g * 0.5 ** 0.5))
    return 0.5 * g * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (g + 0.044715 * g * g * g)))


def _gated(s, c):
    a = s["a"].float()
    if c["ln"]:
        a = a - a.mean(1, keepdim=True)
        a = a / torch.sqrt((a * a).mean(1, keepdim=True) + LN_EPS)
    y = torch.matmul(a, s["bt"].float().t())
    if c["bias"]:
        y = y + s["bias"]
    return (_act(y[:, :c["n"]], c["act"]) * y[:, c["n"]:]).to(TORCH[c["dtype"]])


def _logp(s, c):
    x = s["logits"].float()
    m = x.amax(1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    z = e.sum(1, keepdim=True)
    log_z = torch.log(z)
    got = {"logp": torch.gather(d, 1, s["tokens"].long()) - log_z, "lse": (m + log_z)[:, 0],
           "entropy": (log_z - torch.where(e > 0, e * d, torch.zeros_like(d)).sum(1, keepdim=True) / z)[:, 0]}
    if c["k"]:
        # one whole number a logit: its place in the order of values, then the lower index first
        bits = (x + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7fffffff)).long() << 32
        key += (2 ** 31 - 1) - torch.arange(c["vocab"], device="cuda")
        best = torch.topk(key, c["k"], dim=1, sorted=True).values
        at = (2 ** 31 - 1) - (best & 0xffffffff)
        lp = torch.gather(d, 1, at) - log_z
        got["topi"] = torch.where(lp == -math.inf, torch.full_like(at, NONE), at).int()
        got["toplp"] = lp
    return got


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    return {"append": _append, "attn": _attn, "gated": _gated, "logp": _logp}[c["kind"]](state, c)


# ---- the definitions in 64 bits ----------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        page, w = case["page"], case["kv_heads"] * case["d_head"]
        lens, new = _lengths(case)
        table = s["table"].cpu()
        row, src, to, slot = 0, [], [], []
        for b, count in enumerate(new):
            for j in range(count):
                pos = lens[b] - count + j
                src.append(row + j)
                to.append(int(table[b, pos // page]))
                slot.append(pos % page)
            row += count
        got = {}
        for part, name in ((1, "k"), (2, "v")):
            pool = torch.zeros(s[name].shape, dtype=torch.float64, device="cuda")
            x = s["qkv"][torch.tensor(src, device="cuda")].double()[:, part * w:(part + 1) * w]
            if case["fp8"]:
                a = x.abs().clamp(max=448.0)
                step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3.0)    # 3 mantissa bits, subnormals at 2^-9
                x = torch.sign(x) * torch.clamp(torch.round(a / step) * step, max=448.0)    # ties to even
            pool[torch.tensor(to, device="cuda"), :, torch.tensor(slot, device="cuda")] = x.view(
                -1, case["kv_heads"], case["d_head"])
            got[name] = pool
        return got
    if case["kind"] == "attn":
        lens = s["lens"].tolist()
        group = case["heads"] // case["kv_heads"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            if n == 0:
                continue
            at = s["table"][b, :(n + case["page"] - 1) // case["page"]].long()
            for g in range(case["kv_heads"]):
                if case["fp8"]:
                    k, v = (s[x].view(torch.uint8)[at, g].view(torch.float8_e4m3fn).double() for x in "kv")
                else:
                    k, v = (s[x][at, g].double() for x in "kv")
                k, v = k.reshape(-1, case["d_head"])[:n], v.reshape(-1, case["d_head"])[:n]
                q = s["q"][b, g * group:(g + 1) * group].double()
                z = torch.softmax(q @ k.t().contiguous() * s["scale"], 1)
                out[b, g * group:(g + 1) * group] = z @ v
        return out
    if case["kind"] == "gated":
        x, w, n = s["a"].double(), s["bt"].double(), case["n"]
        if case["ln"]:
            var, mean = torch.var_mean(x, dim=1, keepdim=True, unbiased=False)
            x = (x - mean) * torch.rsqrt(var + LN_EPS)
        bias = s["bias"].double() if case["bias"] else torch.zeros(2 * n, dtype=torch.float64, device="cuda")
        gate, up = x @ w[:n].t().contiguous() + bias[:n], x @ w[n:].t().contiguous() + bias[n:]
        if case["act"] == "relu":
            gate = torch.relu(gate)
        elif case["act"] == "silu":
            gate = gate * torch.sigmoid(gate)
        else:
            gate = torch.nn.functional.gelu(gate, approximate="tanh" if case["act"] == "gelu_tanh" else "none")
        return gate * up
    parts = []
    for i in range(0, case["rows"], 256):
        lp = torch.log_softmax(s["logits"][i:i + 256].double(), 1)
        p = lp.exp()
        part = {"logp": lp.gather(1, s["tokens"][i:i + 256].long()), "lse": torch.logsumexp(s["logits"][i:i + 256].double(), 1),
                "entropy": -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)}
        if case["k"]:
            v, at = torch.sort(s["logits"][i:i + 256].float(), dim=1, descending=True, stable=True)
            at = at[:, :case["k"]]
            part["topi"] = torch.where(v[:, :case["k"]] == -math.inf, torch.full_like(at, NONE), at).int()
            part["toplp"] = lp.gather(1, at)
        parts.append(part)
    return {n: torch.cat([p[n] for p in parts]) for n in parts[0]}
