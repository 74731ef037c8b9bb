"""What a request goes through around its decoder steps, as timed and compared cases: pages for its
tokens, attention over its prompt, attention for the tokens drafted ahead of it, and the drafted
tokens that stay.

Four kinds of case, each calls of entry points of ``paper_2109_08008_amd.nt``:

* ``resize``  block tables, positions and slots from the requests' lengths: a growth and the return
              of the same tokens, ``nt_op_kv_resize`` twice;
* ``prompt``  attention over whole packed sequences, ``nt_op_attn_prompt``;
* ``tree``    attention of several new tokens a sequence over a paged cache, which see the context and
              a tree (or a chain) of each other, ``nt_op_attn_tree``;
* ``keep``    the accepted drafted tokens' keys and values moved behind the context, ``nt_op_kv_keep``.

``run`` computes them in elementary torch operations (``own`` false) or through the library.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
MAX_CACHE = 1 << 29      # n_seqs * longest * kv_heads * d_head of a drawn cache
MAX_SCORES = 1 << 31     # scores that a plain form holds at once
MAX_PAIRS = 16 * 8192 * 8192     # heads * (query, key) pairs of a drawn call
MAX_ROWS = 1 << 21


def listed():
    return [
        # a decoder step of 96 live hypotheses: most stay on their page
        {"name": "resize_step", "kind": "resize", "n_seqs": 96, "page": 16, "shortest": 1, "longest": 160, "new_min": 1,
         "new_max": 1, "pad": 0},
        # 4096 requests of a server's queue arrive at once with prompts of up to a few hundred tokens
        {"name": "resize_prompts", "kind": "resize", "n_seqs": 4096, "page": 64, "shortest": 0, "longest": 0, "new_min": 1,
         "new_max": 900, "pad": 1000},
        # one short prompt: latency counts
        {"name": "prompt_one", "kind": "prompt", "dtype": "f16", "n_seqs": 1, "heads": 8, "kv_heads": 8, "d_head": 64,
         "shortest": 77, "longest": 77, "causal": True},
        # a batch of 540 packed source sentences of up to 150 tokens in a wide encoder: no padding, no mask
        {"name": "prompt_sentences", "kind": "prompt", "dtype": "f16", "n_seqs": 540, "heads": 16, "kv_heads": 16,
         "d_head": 64, "shortest": 1, "longest": 150, "causal": False},
        # documents of different lengths, four query heads to a key head, bf16
        {"name": "prompt_documents_bf16", "kind": "prompt", "dtype": "bf16", "n_seqs": 8, "heads": 32, "kv_heads": 8,
         "d_head": 128, "shortest": 500, "longest": 8000, "causal": True},
        # one long document
        {"name": "prompt_long", "kind": "prompt", "dtype": "f16", "n_seqs": 1, "heads": 16, "kv_heads": 16, "d_head": 128,
         "shortest": 16383, "longest": 16383, "causal": True},
        # eight drafted tokens for each of four sentences: latency counts
        {"name": "tree_sentences", "kind": "tree", "dtype": "f16", "fp8": False, "n_seqs": 4, "heads": 8, "kv_heads": 8,
         "d_head": 64, "page": 16, "shortest": 5, "longest": 60, "new_min": 8, "new_max": 8, "tree": True},
        # trees of up to 24 drafted tokens for 64 requests, four query heads to a key head, bf16
        {"name": "tree_batch_bf16", "kind": "tree", "dtype": "bf16", "fp8": False, "n_seqs": 64, "heads": 32, "kv_heads": 8,
         "d_head": 128, "page": 32, "shortest": 100, "longest": 4000, "new_min": 1, "new_max": 24, "tree": True},
        # one request with a very long FP8 cache and a full tree: only the split over its length fills the GPU
        {"name": "tree_long_fp8", "kind": "tree", "dtype": "f16", "fp8": True, "n_seqs": 1, "heads": 16, "kv_heads": 4,
         "d_head": 128, "page": 128, "shortest": 131001, "longest": 131001, "new_min": 64, "new_max": 64, "tree": True},
        # prompts that come in pieces: the next few hundred tokens of 12 requests behind what is cached
        {"name": "tree_pieces", "kind": "tree", "dtype": "f16", "fp8": False, "n_seqs": 12, "heads": 16, "kv_heads": 4,
         "d_head": 128, "page": 64, "shortest": 1000, "longest": 8000, "new_min": 200, "new_max": 500, "tree": False},
        # the accepted branch of 64 requests' trees
        {"name": "keep_step", "kind": "keep", "dtype": "f16", "fp8": False, "n_seqs": 64, "kv_heads": 8, "d_head": 128,
         "page": 32, "shortest": 100, "longest": 600, "new_min": 1, "new_max": 24},
        # many requests with full trees and long accepted branches, bf16
        {"name": "keep_many_bf16", "kind": "keep", "dtype": "bf16", "fp8": False, "n_seqs": 900, "kv_heads": 8, "d_head": 128,
         "page": 64, "shortest": 64, "longest": 300, "new_min": 48, "new_max": 64},
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("resize", "prompt", "prompt", "prompt", "tree", "tree", "tree", "keep"))
    if kind == "resize":
        c = {"kind": kind, "n_seqs": spread(1, 8192), "page": rng.choice((16, 32, 64, 128, 256))}
        c["shortest"] = rng.choice((0, 1, 300))
        c["longest"] = c["shortest"] + spread(1, 2000)
        c["new_min"] = rng.choice((0, 1))
        c["new_max"] = 1 if rng.random() < 0.4 else spread(2, max(2, min(4000, MAX_ROWS // c["n_seqs"])))
        c["pad"] = rng.choice((0, 1, 77, 4096))
        return c
    dtype = rng.choice(("f16", "f16", "bf16", "bf16", "f32"))
    c = {"kind": kind, "dtype": dtype}
    if kind == "prompt":
        c["kv_heads"] = rng.choice((1, 2, 3, 4, 8, 16))
        c["heads"] = c["kv_heads"] * rng.choice((1, 1, 2, 3, 4, 8))
        c["d_head"] = rng.choice((32, 64, 64, 128, 128))
        c["n_seqs"] = spread(1, 600)
        c["longest"] = spread(1, 16000)
        limit = MAX_PAIRS // (8 if dtype == "f32" else 1)
        while c["heads"] * c["n_seqs"] * c["longest"] ** 2 > limit or c["n_seqs"] * c["longest"] > 1 << 17:
            c["n_seqs"], c["longest"] = max(1, c["n_seqs"] * 2 // 3), max(1, c["longest"] * 4 // 5)
        c["shortest"] = max(1, int(c["longest"] * rng.choice((0.01, 0.3, 1.0))))
        c["causal"] = rng.random() < 0.7
        return c
    c["fp8"] = dtype == "f16" and rng.random() < 0.4
    c["kv_heads"] = rng.choice((1, 2, 3, 4, 8, 16))
    c["d_head"] = rng.choice((32, 64, 128))
    c["page"] = rng.choice((16, 32, 64, 128, 256))
    width = c["kv_heads"] * c["d_head"]
    if kind == "keep":
        c["n_seqs"] = spread(1, 1024)
        c["new_min"] = 1
        c["new_max"] = spread(2, 64)
        c["shortest"] = rng.choice((0, 10, 200))
        c["longest"] = c["shortest"] + spread(1, 2000)
        while c["n_seqs"] * (c["longest"] + c["new_max"] + c["page"]) * width > MAX_CACHE // 2:
            c["n_seqs"], c["longest"] = (c["n_seqs"] + 1) // 2, c["shortest"] + (c["longest"] - c["shortest"] + 1) // 2
        return c
    c["heads"] = c["kv_heads"] * rng.choice((1, 1, 2, 4, 5, 8))
    c["tree"] = rng.random() < 0.7
    c["new_max"] = spread(1, 64) if c["tree"] else spread(2, 1000)
    c["new_min"] = rng.choice((1, 1, c["new_max"]))
    c["n_seqs"] = spread(1, 512)
    c["longest"] = c["new_max"] + spread(1, 100000)
    limit = MAX_PAIRS // (8 if dtype == "f32" else 1)
    while (c["n_seqs"] * (c["longest"] + c["page"]) * width > MAX_CACHE
           or c["n_seqs"] * c["longest"] * c["new_max"] * c["heads"] > limit):
        c["n_seqs"], c["longest"] = (c["n_seqs"] + 1) // 2, max(c["new_max"] + 1, c["longest"] * 3 // 4)
        if c["n_seqs"] == 1 and c["longest"] == c["new_max"] + 1:
            break
    c["shortest"] = max(c["new_max"], int(c["longest"] * rng.choice((0.01, 0.3, 1.0))))
    if c["n_seqs"] > 8 and rng.random() < 0.3:
        c["new_min"] = 0      # some have no new token in this step
    return c


def _sizes(case):
    """The sequences' lengths (new tokens included) and new tokens: the case's own, whatever the seed."""
    r = random.Random("%(kind)s %(n_seqs)d %(shortest)d %(longest)d" % case)
    n = case["n_seqs"]
    lens = [r.randint(case["shortest"], case["longest"]) for _ in range(n)]
    if case["kind"] == "prompt":
        return lens, lens
    new = [r.randint(case["new_min"], case["new_max"]) for _ in range(n)]
    if case["kind"] == "tree":
        if n > 8:
            lens[r.randrange(n)] = case["new_max"]      # nothing cached yet
        return lens, [min(a, b) for a, b in zip(new, lens)]
    return [a + b for a, b in zip(lens, new)], new


def _parents(case, new):
    """Each drafted token's parent among its sequence's drafted tokens, -1 for the context's last token."""
    r = random.Random("parents %(n_seqs)d %(new_max)d %(longest)d" % case)
    return [[r.randint(max(-1, i - 6), i - 1) for i in range(n)] for n in new]


def _masks(case, new):
    """For each new token of a tree, the bits of the new tokens that it sees: itself and its ancestors."""
    got = []
    for parents in _parents(case, new):
        seen = []
        for i, p in enumerate(parents):
            seen.append((1 << i) | (seen[p] if p >= 0 else 0))
        got += seen
    return got


def _branches(case, new):
    """The accepted tokens of each sequence: the first ones of its main branch (the drafted tokens come in
    depth-first order, half of them on that branch), then some of a side branch."""
    r = random.Random("branches %(n_seqs)d %(new_max)d %(longest)d" % case)
    got = []
    for n in new:
        deep = (n + 1) // 2
        most = r.randint(0, deep)
        main = r.randint(0, most)
        path = list(range(main))
        rest = range(deep, n)
        path += sorted(r.sample(rest, min(most - main, len(rest))))
        got.append(path)
    return got


def _cell(case):
    return 1 if case.get("fp8") else BYTES[case["dtype"]]


def work(case):
    """Bytes and operations that one pass cannot do without: inputs read once, outputs written once."""
    lens, new = _sizes(case)
    n = case["n_seqs"]
    if case["kind"] == "resize":
        grown = sum((a + case["page"] - 1) // case["page"] - (a - b + case["page"] - 1) // case["page"]
                    for a, b in zip(lens, new))
        # lengths, counts and offsets; each page's entry and place in the ring, there and back; a position and a slot
        return {"bytes": float(n * 28 + 16 * grown + 12 * (sum(new) + case["pad"])), "flops": 0.0}
    if case["kind"] == "keep":
        moved = sum(sum(i != at for i, at in enumerate(path)) for path in _branches(case, new))
        return {"bytes": float(moved * 4 * case["kv_heads"] * case["d_head"] * _cell(case) + n * 16), "flops": 0.0}
    h, hkv, dh, eb = case["heads"], case["kv_heads"], case["d_head"], BYTES[case["dtype"]]
    if case["kind"] == "prompt":
        pairs = sum(a * (a + 1) // 2 if case["causal"] else a * a for a in lens)
        return {"bytes": float(sum(lens) * 2 * (h + hkv) * dh * eb), "flops": 4.0 * pairs * h * dh}
    if case["tree"]:
        pairs = sum((a - b) * b for a, b in zip(lens, new)) + sum(bin(x).count("1") for x in _masks(case, new))
    else:
        pairs = sum((a - b) * b + b * (b + 1) // 2 for a, b in zip(lens, new))
    return {"bytes": float(sum(a for a, b in zip(lens, new) if b) * 2 * hkv * dh * _cell(case)
                           + sum(new) * (2 * h * dh * eb + 8)),
            "flops": 4.0 * pairs * h * dh}


def _normal(gen, *shape, scale=1.0, shift=0.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(dtype)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _offsets(counts):
    off = [0]
    for x in counts:
        off.append(off[-1] + x)
    return off


def _cache(s, case, gen, seed, lens):
    """Pools, page table and, for the library, the cache over them."""
    hkv, dh, page, n = case["kv_heads"], case["d_head"], case["page"], case["n_seqs"]
    need = [(x + page - 1) // page for x in lens]
    most = max(1, max(need))
    n_pages = sum(need) + 3
    order = list(range(n_pages))      # a pool in use for a while: pages lie anywhere
    random.Random(seed).shuffle(order)
    rows, at = [], 0
    for p in need:
        rows.append(order[at:at + p] + [-1] * (most - p))
        at += p
    cell = torch.float8_e4m3fn if case["fp8"] else TORCH[case["dtype"]]
    s["table"] = _ints(rows)
    s["lens"] = _ints(lens)
    for name, shift in (("k", 0.0), ("v", 0.1)):
        s[name] = torch.empty(n_pages, hkv, page, dh, dtype=cell, device="cuda")
        for p in range(0, n_pages, 4096):
            s[name][p:p + 4096] = _normal(gen, *s[name][p:p + 4096].shape, shift=shift).to(cell)
    if own:
        from paper_2109_08008_amd import nt
        s["cache"] = nt.kv_pages(case["dtype"], hkv, dh, page, n_pages, most, s["k"].data_ptr(), s["v"].data_ptr(),
                                 s["table"].data_ptr(), fp8=case["fp8"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens, new = _sizes(case)
    n = case["n_seqs"]
    s = {"case": case}
    if case["kind"] == "resize":
        page = case["page"]
        have = [(a - b + page - 1) // page for a, b in zip(lens, new)]
        s["max_pages"] = max(1, max((a + page - 1) // page for a in lens))
        s["n_pages"] = sum((a + page - 1) // page for a in lens) + 5
        order = list(range(s["n_pages"]))
        random.Random(seed).shuffle(order)
        rows, at = [], 0
        for p in have:
            rows.append(order[at:at + p] + [-1] * (s["max_pages"] - p))
            at += p
        head = random.Random(seed + 1).randrange(s["n_pages"])
        s["table"] = _ints(rows)
        s["ring"] = torch.full((s["n_pages"],), -1, dtype=torch.int32, device="cuda")
        free = order[at:]
        s["ring"][(torch.arange(len(free), device="cuda") + head) % s["n_pages"]] = _ints(free)
        s["state"] = _ints([head, len(free), 0, 0])
        s["lens"] = _ints([a - b for a, b in zip(lens, new)])
        s["add"] = _ints(new)
        s["back"] = -s["add"]
        s["rows"] = sum(new) + case["pad"]      # the step's rows, and those that pad it to a fixed number
        s["off"] = torch.empty(n + 1, dtype=torch.int32, device="cuda")
        s["pos"] = torch.empty(s["rows"], dtype=torch.int32, device="cuda")
        s["slot"] = torch.empty(s["rows"], dtype=torch.int64, device="cuda")
        return s
    dt, hkv, dh = TORCH[case["dtype"]], case["kv_heads"], case["d_head"]
    off = _offsets(new)
    s["off"] = _ints(off)
    if case["kind"] == "prompt":
        h, rows = case["heads"], off[-1]
        # the projection's rows hold query, key and value side by side
        s["qkv"] = _normal(gen, rows, (h + 2 * hkv) * dh, dtype=dt)
        s["qkv"][:, (h + hkv) * dh:] += 0.1
        s["longest"] = max(lens)
        s["out"] = torch.empty(rows, h * dh, dtype=dt, device="cuda")
        s["scale"] = dh ** -0.5
        return s
    _cache(s, case, gen, seed, lens)
    if case["kind"] == "keep":
        paths = _branches(case, new)
        most = max(1, max(len(p) for p in paths))
        s["path"] = _ints([p + [-1] * (most - len(p)) for p in paths])
        s["n_path"] = _ints([len(p) for p in paths])
        s["add"] = torch.empty(n, dtype=torch.int32, device="cuda")
        return s
    h, rows = case["heads"], off[-1]
    s["q"] = _normal(gen, max(rows, 1), h * dh, dtype=dt)
    s["out"] = torch.zeros(max(rows, 1), h * dh, dtype=dt, device="cuda")
    s["rows"], s["max_new"], s["max_len"], s["scale"] = rows, max(new), max(lens), dh ** -0.5
    # 64 bits a row, the highest one a sign for torch
    s["mask"] = _ints([x - (1 << 64) if x >> 63 else x for x in _masks(case, new)] or [0], torch.int64) if case["tree"] else None
    if own:
        from paper_2109_08008_amd import nt
        need = nt.nt_op_attn_tree_workspace(s["cache"], h, n, rows, s["max_new"], s["max_len"])
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return s


def _run_own(s):
    from paper_2109_08008_amd import nt
    c = s["case"]
    n = c["n_seqs"]
    if c["kind"] == "resize":
        nt.nt_op_kv_resize(c["page"], s["n_pages"], s["max_pages"], s["table"].data_ptr(), s["lens"].data_ptr(),
                           s["add"].data_ptr(), n, s["ring"].data_ptr(), s["state"].data_ptr(), s["off"].data_ptr(),
                           s["pos"].data_ptr(), s["slot"].data_ptr(), s["rows"])
        nt.nt_op_kv_resize(c["page"], s["n_pages"], s["max_pages"], s["table"].data_ptr(), s["lens"].data_ptr(),
                           s["back"].data_ptr(), n, s["ring"].data_ptr(), s["state"].data_ptr(), None, None, None, 0)
        return {x: s[x] for x in ("table", "lens", "ring", "state", "off", "pos", "slot")}
    if c["kind"] == "prompt":
        w, eb, base = c["d_head"], BYTES[c["dtype"]], s["qkv"].data_ptr()
        ld = s["qkv"].shape[1]
        nt.nt_op_attn_prompt(c["dtype"], base, ld, c["heads"], base + c["heads"] * w * eb,
                             base + (c["heads"] + c["kv_heads"]) * w * eb, ld, c["kv_heads"], w, s["off"].data_ptr(), n,
                             s["qkv"].shape[0], c["causal"], s["scale"], s["out"].data_ptr(), c["heads"] * w)
        return s["out"]
    if c["kind"] == "tree":
        w = c["heads"] * c["d_head"]
        nt.nt_op_attn_tree(s["cache"], s["q"].data_ptr(), w, c["heads"], s["off"].data_ptr(),
                           s["mask"].data_ptr() if c["tree"] else None, s["lens"].data_ptr(), n, s["rows"], s["max_new"],
                           s["max_len"], s["scale"], s["out"].data_ptr(), w, s["ws"].data_ptr(), s["ws"].numel())
        return s["out"]
    nt.nt_op_kv_keep(s["cache"], s["off"].data_ptr(), s["lens"].data_ptr(), s["path"].data_ptr(), s["path"].shape[1],
                     s["n_path"].data_ptr(), n, s["add"].data_ptr())
    return {"k": s["k"], "v": s["v"], "add": s["add"]}


# ---- plain forms -------------------------------------------------------------------------
def _resize_once(s, c, add):
    page, ring_len = c["page"], s["n_pages"]
    lens = s["lens"].long()
    new = torch.clamp(lens + add.long(), min=0)
    have, need = (lens + page - 1) // page, (new + page - 1) // page
    grow, give = torch.clamp(need - have, min=0), torch.clamp(have - need, min=0)
    head, count = s["state"][0].long(), s["state"][1].long()
    short = torch.clamp(grow.sum() - count, min=0)
    j = torch.arange(s["max_pages"], device="cuda")[None, :]
    table = s["table"].long()
    first = torch.cumsum(grow, 0) - grow
    taken = (j >= have[:, None]) & (j < need[:, None])
    page_of = s["ring"].long()[(head + first[:, None] + j - have[:, None]) % ring_len]
    given = (j >= need[:, None]) & (j < have[:, None])
    back = (head + count + (torch.cumsum(give, 0) - give)[:, None] + j - need[:, None]) % ring_len
    spare = torch.cat([s["ring"], s["ring"][:1]])
    spare.scatter_(0, torch.where(given, back, torch.full_like(back, ring_len)).reshape(-1), s["table"].reshape(-1))
    s["ring"].copy_(spare[:ring_len])
    s["table"].copy_(torch.where(taken, page_of, torch.where(given, torch.full_like(table, -1), table)))
    s["lens"].copy_(new)
    rows = torch.clamp(add.long(), min=0)
    s["state"].copy_(torch.stack([(head + grow.sum()) % ring_len, count - grow.sum() + give.sum(), short, rows.sum()]))
    return lens, rows


def _resize(s, c):
    lens, rows = _resize_once(s, c, s["add"])
    ends = torch.cumsum(rows, 0)
    s["off"][0] = 0
    s["off"][1:] = ends
    at = torch.arange(s["rows"], device="cuda")
    seq = torch.clamp(torch.searchsorted(ends, at, right=True), max=c["n_seqs"] - 1)
    real = at < ends[-1]
    pos = lens[seq] + at - (ends[seq] - rows[seq])
    slot = s["table"].long()[seq, torch.clamp(pos // c["page"], max=s["max_pages"] - 1)] * c["page"] + pos % c["page"]
    none = torch.full_like(pos, -1)
    s["pos"].copy_(torch.where(real, pos, none))
    s["slot"].copy_(torch.where(real, slot, none))
    _resize_once(s, c, s["back"])
    return {x: s[x] for x in ("table", "lens", "ring", "state", "off", "pos", "slot")}


def _softmax(x, seen):
    """Softmax over the last axis, in place; a row that sees nothing is zero."""
    x.masked_fill_(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    x.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    z = x.sum(-1, keepdim=True)
    return x.div_(torch.where(z == 0, torch.ones_like(z), z))


def _prompt(s, c):
    n, h, hkv, dh, length = c["n_seqs"], c["heads"], c["kv_heads"], c["d_head"], s["longest"]
    off = s["off"].long()
    rows = s["qkv"].shape[0]
    at = torch.arange(length, device="cuda")
    step = max(1, MAX_SCORES // (h * length * length))
    seq = torch.searchsorted(off[1:], torch.arange(rows, device="cuda"), right=True)
    padded = torch.empty(n, length, h * dh, dtype=torch.float32, device="cuda")
    for b in range(0, n, step):      # as many sequences as fit
        e = min(n, b + step)
        x = s["qkv"][torch.clamp(off[b:e, None] + at, max=rows - 1)].float()
        q = x[..., :h * dh].reshape(e - b, length, hkv, h // hkv, dh).permute(0, 2, 3, 1, 4)
        k = x[..., h * dh:(h + hkv) * dh].reshape(e - b, length, hkv, dh).permute(0, 2, 3, 1).contiguous()
        v = x[..., (h + hkv) * dh:].reshape(e - b, length, hkv, dh).permute(0, 2, 1, 3).contiguous()
        p = torch.matmul((q * s["scale"]).reshape(e - b, hkv, -1, dh), k).reshape(e - b, hkv, h // hkv, length, length)
        seen = at < (off[b + 1:e + 1] - off[b:e])[:, None]
        seen = seen[:, None, None, None, :]
        if c["causal"]:
            seen = seen & (at[None, :] <= at[:, None])
        p = _softmax(p, seen).reshape(e - b, hkv, -1, length)
        o = torch.matmul(p, v).reshape(e - b, h, length, dh)
        padded[b:e] = o.permute(0, 2, 1, 3).reshape(e - b, length, h * dh)
        del p, o, q, k, v, x
    return padded[seq, torch.arange(rows, device="cuda") - off[seq]].to(TORCH[c["dtype"]])


def _tree(s, c):
    n, h, hkv, dh, most = c["n_seqs"], c["heads"], c["kv_heads"], c["d_head"], max(1, s["max_new"])
    at = s["table"].long().clamp(min=0)
    length = at.shape[1] * c["page"]
    off, lens = s["off"].long(), s["lens"].long()
    new = off[1:] - off[:-1]

    def keys(pool):     # [n, hkv, length, dh]
        x = pool.view(torch.uint8)[at].view(torch.float8_e4m3fn).float() if c["fp8"] else pool[at].float()
        return x.permute(0, 2, 1, 3, 4).reshape(n, hkv, length, dh)

    i = torch.arange(most, device="cuda")
    row = torch.clamp(off[:-1, None] + i, max=s["q"].shape[0] - 1)
    q = (s["q"][row].float() * s["scale"]).reshape(n, most, hkv, h // hkv, dh)
    q = q.permute(0, 2, 4, 3, 1).reshape(n, hkv, dh, -1).contiguous()        # queries in the last axis
    x = torch.matmul(keys(s["k"]), q).transpose(2, 3).contiguous().reshape(n, hkv, h // hkv, most, length)
    pos = torch.arange(length, device="cuda")
    base = (lens - new)[:, None]
    behind = pos[None, :] - base                    # which new token a position is
    context = (pos[None, :] < base)[:, None, :]
    if c["tree"]:
        bit = (s["mask"][row][:, :, None] >> torch.clamp(behind, 0, 63)[:, None, :]) & 1
        seen = context | ((bit == 1) & ((behind >= 0) & (behind < new[:, None]))[:, None, :])
    else:
        seen = context | ((behind[:, None, :] >= 0) & (behind[:, None, :] <= i[None, :, None]))
    seen = seen & (pos[None, :] < lens[:, None])[:, None, :]
    p = _softmax(x, seen[:, None, None]).reshape(n, hkv, -1, length)
    o = torch.matmul(p, keys(s["v"])).reshape(n, h, most, dh).permute(0, 2, 1, 3).reshape(n, most, h * dh)
    rows = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(off[1:], rows, right=True)
    s["out"][:s["rows"]] = o[seq, rows - off[seq]].to(s["out"].dtype)
    return s["out"]


def _keep(s, c):
    off, lens, path = s["off"].long(), s["lens"].long(), s["path"].long()
    new = off[1:] - off[:-1]
    base = (lens - new)[:, None]
    i = torch.arange(path.shape[1], device="cuda")[None, :]
    some = i < s["n_path"].long()[:, None]
    seq = torch.arange(c["n_seqs"], device="cuda")[:, None].expand_as(path)
    src, dst = base + torch.where(some, path, torch.zeros_like(path)), base + i
    # a place that nothing goes to takes what it has
    dst = torch.where(some, dst, src)
    src, dst, seq = src.reshape(-1), dst.reshape(-1), seq.reshape(-1)
    live = some.reshape(-1)
    src, dst, seq = src[live], dst[live], seq[live]
    table = s["table"].long()
    for name in ("k", "v"):
        pool = s[name].view(torch.uint8) if c["fp8"] else s[name]
        pool[table[seq, dst // c["page"]], :, dst % c["page"]] = pool[table[seq, src // c["page"]], :, src % c["page"]]
    s["add"].copy_(s["n_path"].long() - new)
    return {"k": s["k"], "v": s["v"], "add": s["add"]}


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    return {"resize": _resize, "prompt": _prompt, "tree": _tree, "keep": _keep}[c["kind"]](state, c)


# ---- the definitions in 64 bits ----------------------------------------------------------
def _attend(q, k, v, scale, seen):
    """[heads, rows, dh] of one key head's queries, a few of them at a time."""
    out = torch.zeros_like(q)
    step = max(1, (1 << 28) // max(1, q.shape[1] * k.shape[0]))
    kt = k.t().contiguous()
    for i in range(0, q.shape[0], step):
        x = torch.matmul(q[i:i + step], kt) * scale
        if seen is not None:
            x = x.masked_fill(~seen, -math.inf)
        out[i:i + step] = torch.nan_to_num(torch.softmax(x, -1)) @ v
    return out


def exact(case, seed):
    if case["kind"] == "resize":
        return None      # whole numbers only
    s = prepare(case, seed)
    lens, new = _sizes(case)
    if case["kind"] == "keep":
        got = {"k": s["k"].float().double() if case["fp8"] else s["k"].double(),
               "v": s["v"].float().double() if case["fp8"] else s["v"].double(), "add": None}
        table = s["table"].tolist()
        page, to, source = case["page"], [], []
        for b, path in enumerate(_branches(case, new)):
            base = lens[b] - new[b]
            for i, at in enumerate(path):
                to.append((table[b][(base + i) // page], (base + i) % page))
                source.append((table[b][(base + at) // page], (base + at) % page))
        if to:
            a, b = torch.tensor(to, device="cuda").t(), torch.tensor(source, device="cuda").t()
            for name in ("k", "v"):
                got[name][a[0], :, a[1]] = got[name][b[0], :, b[1]]
        return got
    h, hkv, dh = case["heads"], case["kv_heads"], case["d_head"]
    group, off = h // hkv, _offsets(new)
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    masks, first = _masks(case, new) if case.get("tree") else None, 0
    for b, rows in enumerate(new):
        if rows == 0:
            continue
        base = 0 if case["kind"] == "prompt" else lens[b] - rows
        if case["kind"] == "prompt":
            seen = torch.ones(rows, rows, dtype=torch.bool, device="cuda").tril_() if case["causal"] else None
        else:
            seen = torch.ones(rows, lens[b], dtype=torch.bool, device="cuda")
            if case["tree"]:
                bits = [[x >> j & 1 for j in range(rows)] for x in masks[first:first + rows]]
                seen[:, base:] = torch.tensor(bits, device="cuda") == 1
            else:
                seen[:, base:] = seen[:, base:].tril()
            at = s["table"][b, :(lens[b] + case["page"] - 1) // case["page"]].long()
        for g in range(hkv):
            if case["kind"] == "prompt":
                x = s["qkv"][off[b]:off[b + 1]].double()
                q, k, v = x[:, g * group * dh:(g + 1) * group * dh], x[:, (h + g) * dh:][:, :dh], x[:, (h + hkv + g) * dh:][:, :dh]
            else:
                q = s["q"][off[b]:off[b + 1], g * group * dh:(g + 1) * group * dh].double()
                if case["fp8"]:
                    k, v = (s[x].view(torch.uint8)[at, g].view(torch.float8_e4m3fn).double() for x in "kv")
                else:
                    k, v = (s[x][at, g].double() for x in "kv")
                k, v = k.reshape(-1, dh)[:lens[b]], v.reshape(-1, dh)[:lens[b]]
            q = q.reshape(rows, group, dh).transpose(0, 1).contiguous()
            o = _attend(q, k, v.contiguous(), s["scale"], seen)
            out[off[b]:off[b + 1], g * group * dh:(g + 1) * group * dh] = o.transpose(0, 1).reshape(rows, group * dh)
        first += rows
    return out
