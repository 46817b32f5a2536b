"""Cases of the operators around the verify step's cache and logits: keys and values rotated and appended to the paged cache (16 bits, or
8 bits with a power-of-two scale for each page and head), tree attention over the 8-bit cache, the commit of accepted rows in
it, and log probabilities of drafted tokens with entropy and alternatives.

`own` false: the plain forms, elementary torch operations in 32 bits.  `own` true: the framework's entry points.

An 8-bit block is one page of one head: 128-element rows of e4m3 values v that stand for v * 2^e, with e a whole number in [-24, 7], the
smallest for which the block's largest magnitude is at most 448 * 2^e (beyond 448 * 2^7 values saturate)."""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
D = 128
E_MIN, E_MAX, TOP8 = -24, 7, 448.0
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------------------ cases
def _append(name, cache, dtype, batch, nodes, ctx_lo, ctx_hi, hq, hkv, page):
    return {"name": name, "op": "append", "cache": cache, "dtype": dtype, "batch": batch, "nodes": nodes, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "hq": hq, "hkv": hkv, "page": page}


def _attn(name, dtype, batch, kind, nodes, ctx_lo, ctx_hi, hq, hkv, page):
    return {"name": name, "op": "attn", "dtype": dtype, "batch": batch, "kind": kind, "nodes": nodes, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "hq": hq, "hkv": hkv, "page": page}


def _commit(name, batch, nodes, ctx_lo, ctx_hi, hkv, page):
    return {"name": name, "op": "commit", "batch": batch, "nodes": nodes, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "hkv": hkv, "page": page}


def _logprobs(name, dtype, batch, nodes, vocab, top):
    return {"name": name, "op": "logprobs", "dtype": dtype, "batch": batch, "nodes": nodes, "vocab": vocab, "top": top}


def listed():
    return [
        # a drafted chain of 8 after a 2K context, one 8B-shaped layer: the call whose latency counts in every step
        _append("append chain of 8", "16", "bf16", 1, 8, 2048, 2048, 32, 8, 16),
        # a serving batch's drafted trees into the 8-bit cache, contexts that end inside pages
        _append("append 16 trees, 8 bit", "8", "bf16", 16, 32, 4099, 60013, 32, 8, 16),
        # a prompt into an empty 8-bit cache, one token short of a whole number of pages
        _append("append prompt 8191, 8 bit", "8", "bf16", 1, 8191, 0, 0, 32, 8, 16),
        # four prompts of 70B-shaped heads in fp16 behind cached prefixes, larger pages
        _append("append 4 prompts, fp16", "16", "f16", 4, 2047, 1000, 5003, 64, 8, 64),
        # the chain's attention at 2K: latency
        _attn("attn chain, 2K", "bf16", 1, "chain", 8, 2048, 2048, 32, 8, 16),
        # the single long context with a token tree
        _attn("attn tree 32, 32K", "bf16", 1, "tree", 32, 32768, 32768, 32, 8, 16),
        # the mixed serving batch: chains of 8 and trees of 32 over contexts of 4K to 64K
        _attn("attn 16 mixed, 4K-64K", "bf16", 16, "mixed", 32, 4099, 65521, 32, 8, 16),
        # the largest trees over long contexts, fp16 queries: 256 packed rows for each KV head
        _attn("attn 4 x 64K, tree 64", "f16", 4, "tree", 64, 65536, 65536, 32, 8, 16),
        # the commit after one sequence's step
        _commit("commit tree 32", 1, 32, 32771, 32771, 8, 16),
        # the commit after a batch's step
        _commit("commit 64 trees", 64, 64, 500, 4003, 8, 16),
        # one drafted chain's rows over the 8B vocabulary, five alternatives each
        _logprobs("logprobs 8 rows", "f32", 1, 8, 128256, 5),
        # the rows of four 64-node trees, twenty alternatives each
        _logprobs("logprobs 256 rows", "f32", 4, 64, 128256, 20),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "append", "attn", "attn", "attn", "commit", "logprobs", "logprobs"])
    page = rng.choice([16, 16, 32, 64, 128])
    hkv = rng.choice([1, 2, 4, 8, 8])
    if op == "append":
        hq = hkv * rng.choice([1, 2, 3, 4, 8])
        cache = rng.choice(["16", "8"])
        batch = _log_int(rng, 1, 64)
        tokens = _log_int(rng, 1, 8000 // batch)
        lo = rng.choice([0, _log_int(rng, 1, 20000)])
        return {k: v for k, v in _append("", cache, rng.choice(["bf16", "f16"]), batch, tokens, lo, lo + _log_int(rng, 1, 20000), hq, hkv, page).items()
                if k != "name"}
    if op == "attn":
        kind = rng.choice(["chain", "tree", "mixed"])
        nodes = _log_int(rng, 1, 64)
        group = rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8) if g * max(nodes, 8 if kind == "mixed" else 1) <= 256])
        batch = _log_int(rng, 1, 48)
        hi = _log_int(rng, 1, 200000 // batch)
        lo = rng.choice([0, hi, _log_int(rng, 1, hi)])
        return {k: v for k, v in _attn("", rng.choice(["bf16", "f16"]), batch, kind, nodes, lo, hi, group * hkv, hkv, page).items() if k != "name"}
    if op == "commit":
        lo = _log_int(rng, 1, 4000)
        return {k: v for k, v in _commit("", _log_int(rng, 1, 64), _log_int(rng, 1, 64), lo, lo + _log_int(rng, 1, 2000), hkv, page).items() if k != "name"}
    dtype = rng.choice(["f32", "f32", "bf16", "f16"])
    batch = _log_int(rng, 1, 16)
    return {k: v for k, v in _logprobs("", dtype, batch, _log_int(rng, 1, 250 // batch), _log_int(rng, 30, 131001), rng.choice([0, 1, 3, 5, 8, 20, 32])).items()
            if k != "name"}


# ------------------------------------------------------------------------------------------------------------ shapes of a case
def _lens(c):
    return np.linspace(c["ctx_lo"], c["ctx_hi"], c["batch"]).astype(np.int64)


def _counts(c):
    if c.get("kind") == "mixed":                 # every other sequence verifies a chain of 8
        return np.where(np.arange(c["batch"]) % 2 == 0, c["nodes"], min(8, c["nodes"]))
    return np.full(c["batch"], c["nodes"])


def work(c):
    if c["op"] == "logprobs":
        rows = c["batch"] * c["nodes"]
        return {"bytes": rows * (c["vocab"] * (4 if c["dtype"] == "f32" else 2) + 12 + 8 * c["top"]), "flops": 6 * rows * c["vocab"]}
    n, lens = _counts(c), _lens(c)
    total = int(n.sum())
    if c["op"] == "append":
        kv = total * c["hkv"] * D * 2
        return {"bytes": kv * 2 + kv * (2 if c["cache"] == "16" else 1) + 2 * total * c["hq"] * D * 2 + total * D * 4,
                "flops": 3 * total * (c["hq"] + c["hkv"]) * D}
    if c["op"] == "attn":
        keys = int((lens + n).sum())
        pages = int(((lens + n + c["page"] - 1) // c["page"]).sum())
        rows = n * (c["hq"] // c["hkv"])
        return {"bytes": keys * c["hkv"] * 2 * D + pages * (2 * c["hkv"] + 4) + 2 * total * c["hq"] * D * 2 + total * c["hq"] * 4,
                "flops": int((rows * (lens + n)).sum()) * c["hkv"] * 4 * D}
    moved = max(1, min(c["nodes"], 6))           # accepted rows that leave their place, about
    return {"bytes": c["batch"] * moved * c["hkv"] * 4 * D + c["batch"] * 300, "flops": 2 * c["batch"] * moved * c["hkv"] * D}


# ------------------------------------------------------------------------------------------------------------ 8-bit blocks
def _need(amax):
    """The exponent that a largest magnitude needs, from its bits: 448 is 1.75 * 2^8."""
    return (((amax.float().contiguous().view(torch.int32) + 0x1FFFFF) >> 23) - 135).clamp(E_MIN, E_MAX)


def _two(e):
    """2^e in 32 bits, from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(x, e):
    """The e4m3 values of x * 2^-e, saturated; a NaN stays one."""
    return (x.float() * _two(-e)).clamp(-TOP8, TOP8).to(torch.float8_e4m3fn)


def _magnitude(x):
    return torch.nan_to_num(x.float().abs(), nan=0.0, posinf=math.inf).amax(-1)


# ------------------------------------------------------------------------------------------------------------ inputs
def _parents(kind, counts, rng):
    out = []
    for b, n in enumerate(counts):
        chain = kind == "chain" or (kind == "mixed" and b % 2 == 1)
        par = [-1]
        depth = [0]
        for i in range(1, int(n)):
            p = i - 1 if chain else int(rng.integers(max(0, i - 6), i))
            while not chain and depth[p] >= 8:
                p = par[p]
            par.append(p)
            depth.append(depth[p] + 1)
        out.append(par)
    return out


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device=DEV)


def _paged(c, gen, extra=0):
    """Lengths, offsets and a shuffled page table with room for every sequence's context and drafts."""
    lens, counts = _lens(c), _counts(c)
    pages = (lens + counts + c["page"] - 1) // c["page"]
    width, total = int(pages.max()), int(pages.sum()) + 3
    perm = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    first = np.concatenate([[0], np.cumsum(pages)])[:-1]
    at = torch.as_tensor(first, device=DEV)[:, None] + torch.arange(width, device=DEV)[None, :]
    table = torch.where(torch.arange(width, device=DEV)[None, :] < torch.as_tensor(pages, device=DEV)[:, None], perm[at.clamp(max=total - 1)],
                        perm[-1])             # (past a sequence's own pages: one that nobody uses)
    return {"lens": _i32(lens), "offsets": _i32(np.concatenate([[0], np.cumsum(counts)])), "table": table.to(torch.int32).contiguous(), "pages": total,
            "counts": counts, "batch": c["batch"], "total": int(counts.sum()), "most": int(counts.max()), "page": c["page"], "width": width}


def _cache8(c, pages, gen):
    """An 8-bit cache as appends leave it: unit-scale keys and values whose scale differs from head to head."""
    blocks, exps = [], []
    for _ in range(2):
        x = torch.randn((pages, c["hkv"], c["page"], D), generator=gen, device=DEV)
        x *= torch.exp2(torch.randint(-2, 3, (1, c["hkv"], 1, 1), generator=gen, device=DEV).float()) * 0.75
        e = _need(_magnitude(x).amax(-1))
        blocks.append(_encode(x, e[:, :, None, None]))
        exps.append(e)
    return blocks[0], blocks[1], torch.stack(exps, -1).to(torch.int8).contiguous()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    s = {"case": c}
    if c["op"] == "logprobs":
        rows = c["batch"] * c["nodes"]
        s["offsets"] = _i32(np.arange(c["batch"] + 1) * c["nodes"])
        par = _parents("tree", [c["nodes"]] * c["batch"], rng)
        s["parent"] = _i32(np.concatenate(par))
        s["logits"] = (2.0 * torch.randn((rows, c["vocab"]), generator=gen, device=DEV)).to(TYPES[c["dtype"]])
        s["tokens"] = torch.randint(0, c["vocab"], (rows,), generator=gen, device=DEV, dtype=torch.int32)
        # drafted tokens are mostly likely ones: raised at their parents' rows
        base = np.repeat(np.arange(c["batch"]) * c["nodes"], c["nodes"])
        flat = np.concatenate(par)
        hit = np.flatnonzero((flat >= 0) & (rng.random(rows) < 0.6))
        s["logits"][torch.as_tensor((base + flat)[hit], device=DEV), s["tokens"][torch.as_tensor(hit, device=DEV)].long()] += 10
        f = lambda *shape: torch.zeros(shape, dtype=torch.float32, device=DEV)  # noqa: E731
        s["out"] = {"logprob": f(rows), "entropy": f(rows), "lse": f(rows), "top_ids": torch.zeros((rows, c["top"]), dtype=torch.int32, device=DEV),
                    "top_logprobs": f(rows, c["top"])}
        if own:
            from paper_2510_07535_b200 import OwlContext, make_dims
            s["dims"] = make_dims(batch=c["batch"], total_nodes=rows, max_nodes=c["nodes"], vocab=c["vocab"])
            s["ctx"] = OwlContext(s["dims"], torch.device(DEV, torch.cuda.current_device()))
        return s
    s.update(_paged(c, gen))
    n = s["total"]
    if c["op"] == "append":
        t = TYPES[c["dtype"]]
        # one fused projection's output, as a model has it: rows of Hq + 2 Hkv heads
        s["qkv"] = torch.randn((n, c["hq"] + 2 * c["hkv"], D), generator=gen, device=DEV).to(t)
        index = np.concatenate([np.arange(k) for k in s["counts"]])
        depth = index if c["nodes"] > 64 else np.minimum(index, 8)
        s["positions"] = _i32(np.repeat(_lens(c), s["counts"]) + depth)
        rows = int(_lens(c).max() + s["most"])
        angle = torch.arange(rows, device=DEV, dtype=torch.float64)[:, None] * (500000.0 ** (-torch.arange(64, device=DEV, dtype=torch.float64) / 64))
        s["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        if c["cache"] == "8":
            s["k"], s["v"], s["exp"] = _cache8(c, s["pages"], gen)
        else:
            shape = (s["pages"], c["hkv"], c["page"], D)
            s["k"] = torch.randn(shape, generator=gen, device=DEV).to(t)
            s["v"] = torch.randn(shape, generator=gen, device=DEV).to(t)
        s["q_out"] = torch.zeros((n, c["hq"], D), dtype=t, device=DEV)
    elif c["op"] == "attn":
        t = TYPES[c["dtype"]]
        s["q"] = torch.randn((n, c["hq"], D), generator=gen, device=DEV).to(t)
        s["scale"] = 1.0 / math.sqrt(D)
        s["k"], s["v"], s["exp"] = _cache8(c, s["pages"], gen)
        s["parent"] = _i32(np.concatenate(_parents(c["kind"], s["counts"], rng)))
        s["out"] = torch.zeros((n, c["hq"], D), dtype=t, device=DEV)
        s["lse"] = torch.zeros((n, c["hq"]), dtype=torch.float32, device=DEV)
    else:
        s["k"], s["v"], s["exp"] = _cache8(c, s["pages"], gen)
        path, length = np.full((c["batch"], 64), -1), np.zeros(c["batch"])
        for b, par in enumerate(_parents("tree", s["counts"], rng)):
            node, walk = int(rng.integers(len(par))), []
            while node >= 0:
                walk.append(node)
                node = par[node]
            path[b, :len(walk)] = walk[::-1]
            length[b] = len(walk)
        s["path"], s["accepted"] = _i32(path), _i32(length)
    if own:
        from paper_2510_07535_b200 import OwlContext, make_dims
        s["dims"] = make_dims(batch=s["batch"], total_nodes=n, max_nodes=min(64, s["most"]), num_q_heads=c.get("hq", c["hkv"]), num_kv_heads=c["hkv"],
                              page_size=c["page"], max_pages_per_seq=s["width"], num_pages=s["pages"], sm_scale=s.get("scale", 1.0))
        room = make_dims(batch=s["batch"], total_nodes=max(s["batch"], min(n, 64 * s["batch"])), max_nodes=min(64, s["most"]), num_q_heads=c["hkv"],
                         num_kv_heads=c["hkv"], max_pages_per_seq=s["width"], num_pages=s["pages"])
        s["ctx"] = OwlContext(room, torch.device(DEV, torch.cuda.current_device()))
    return s


# ------------------------------------------------------------------------------------------------------------ one pass
def run(s):
    return {"append": _run_append, "attn": _run_attn, "commit": _run_commit, "logprobs": _run_logprobs}[s["case"]["op"]](s)


def _slots(s):
    """For every appended token: its sequence, place in the cache (page, slot)."""
    n, lens = s["total"], s["lens"].long()
    at = torch.arange(n, device=DEV)
    seq = torch.searchsorted(s["offsets"].long(), at, right=True) - 1
    pos = lens[seq] + at - s["offsets"].long()[seq]
    return s["table"].long()[seq, pos // s["page"]], pos % s["page"]


def _rotate(x, cos, sin):
    a, b = x[..., :64].float(), x[..., 64:].float()
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _run_append(s):
    c = s["case"]
    hq, hkv = c["hq"], c["hkv"]
    q, k, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
    if own:
        if c["cache"] == "8":
            s["ctx"].owl_kv_append_fp8(s["dims"], q, k, v, s["positions"], s["rope"], s["q_out"], s["k"], s["v"], s["exp"], s["table"], s["lens"], s["offsets"])
            return [s["q_out"], s["k"], s["v"], s["exp"]]
        s["ctx"].owl_kv_append(s["dims"], q, k, v, s["positions"], s["rope"], s["q_out"], s["k"], s["v"], s["table"], s["lens"], s["offsets"])
        return [s["q_out"], s["k"], s["v"]]
    row = s["rope"][s["positions"].long()][:, None]
    cos, sin = row[..., :64], row[..., 64:]
    s["q_out"].copy_(_rotate(q, cos, sin))
    page, slot = _slots(s)
    new = [_rotate(k, cos, sin), v.float()]
    if c["cache"] == "16":
        s["k"][page, :, slot] = new[0].to(s["k"].dtype)
        s["v"][page, :, slot] = new[1].to(s["v"].dtype)
        return [s["q_out"], s["k"], s["v"]]
    # rows of the context before a sequence's first new token on the same page
    lens = s["lens"].long()
    part = s["table"].long().gather(1, (lens // s["page"]).clamp(max=s["width"] - 1)[:, None])[:, 0]
    old = (torch.arange(s["page"], device=DEV)[None] < (lens % s["page"])[:, None])[:, None, :, None]
    fresh = torch.zeros((s["pages"], 1), dtype=torch.bool, device=DEV)
    fresh[page[slot == 0]] = True
    touched = torch.zeros((s["pages"], 1), dtype=torch.bool, device=DEV)
    touched[page] = True
    after = []
    for i, x in enumerate(new):
        cache, before = s["kv"[i]], s["exp"][..., i].int()
        most = torch.zeros((s["pages"], hkv), device=DEV).scatter_reduce(0, page[:, None].expand(-1, hkv), _magnitude(x), "amax")
        e = torch.where(touched, torch.where(fresh, _need(most), torch.maximum(before, _need(most))), before)
        up = (e - before)[part][:, :, None, None]
        bits = cache.view(torch.uint8)
        was = bits[part]
        kept = _encode(was.view(torch.float8_e4m3fn).float(), up.clamp(min=0))
        bits[part] = torch.where(old & (up > 0), kept.view(torch.uint8), was)
        bits[page, :, slot] = _encode(x, e[page][:, :, None]).view(torch.uint8)
        after.append(e)
    s["exp"].copy_(torch.stack(after, -1))
    return [s["q_out"], s["k"], s["v"], s["exp"]]


def _values(s, cache, exp, dtype):
    """The cache's values, sequence by sequence: [B, Hkv, width * page, D]."""
    t = s["table"].long()
    x = cache.view(torch.uint8)[t].view(torch.float8_e4m3fn).to(dtype)
    x *= _two(exp[t])[..., None, None].to(dtype)
    return x.permute(0, 2, 1, 3, 4).reshape(s["batch"], x.shape[2], -1, D)


def _visible(s):
    """[B, T, keys]: the context, and of the drafted nodes the node's own root path."""
    T, keys = s["most"], s["width"] * s["page"]
    lens, off = s["lens"].long(), s["offsets"].long()
    node = torch.arange(T, device=DEV)
    at = (off[:-1, None] + node[None]).clamp(max=s["total"] - 1)
    real = node[None] < (off[1:] - off[:-1])[:, None]
    par = torch.where(real, s["parent"].long()[at], -1)
    up = (par[..., None] == node).double() + torch.eye(T, device=DEV, dtype=torch.float64)
    anc = (torch.linalg.matrix_power(up, 64) > 0)
    j = torch.arange(keys, device=DEV)[None] - lens[:, None]
    drafted = anc.gather(2, j.clamp(0, T - 1)[:, None].expand(-1, T, -1)) & (j >= 0)[:, None] & (j < T)[:, None]
    return at, real, ((j < 0)[:, None] | drafted) & real[..., None]


def _attention(s, dtype):
    c = s["case"]
    hq, hkv, B, T = c["hq"], c["hkv"], s["batch"], s["most"]
    at, real, sees = _visible(s)
    q = s["q"].to(dtype)[at].view(B, T, hkv, hq // hkv, D).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, D)
    x = (q @ _values(s, s["k"], s["exp"][..., 0], dtype).transpose(2, 3)).mul_(s["scale"])
    mask = sees[:, None, :, None].expand(-1, -1, -1, hq // hkv, -1).reshape(B, 1, -1, x.shape[-1])
    x.masked_fill_(~mask, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    past = torch.arange(s["width"] * s["page"], device=DEV)[None] >= (s["lens"].long() + s["offsets"][1:] - s["offsets"][:-1])[:, None]
    values = _values(s, s["v"], s["exp"][..., 1], dtype).masked_fill_(past[:, None, :, None], 0.0)
    o = ((x @ values) / total).view(B, hkv, T, hq // hkv, D).permute(0, 2, 1, 3, 4).reshape(B, T, hq, D)
    lse = (m + total.log()).view(B, hkv, T, hq // hkv).permute(0, 2, 1, 3).reshape(B, T, hq)
    return o[real], lse[real]


def _run_attn(s):
    if own:
        s["ctx"].owl_verify_attn_fp8(s["dims"], s["q"], s["k"], s["v"], s["exp"], s["table"], s["lens"], s["offsets"], s["parent"], s["out"], s["lse"])
        return [s["out"], s["lse"]]
    out, lse = _attention(s, torch.float32)
    return [out.to(s["q"].dtype), lse]


def _run_commit(s):
    lens = s["lens"].clone()           # the program's committed lengths; the pass moves them on
    if own:
        s["ctx"].owl_kv_commit_fp8(s["dims"], s["k"], s["v"], s["exp"], s["table"], lens, s["offsets"], s["accepted"], s["path"])
        return [s["k"], s["v"], s["exp"], lens]
    hkv, page = s["case"]["hkv"], s["page"]
    L, a, path, table = lens.long()[:, None], s["accepted"].long()[:, None], s["path"].long(), s["table"].long()
    k = torch.arange(64, device=DEV)[None]
    moves = (k < a) & (path != k)
    b, i = moves.nonzero(as_tuple=True)
    start, to = lens.long()[b] + path[b, i], lens.long()[b] + i
    src_page, src_slot = table[b, start // page], start % page
    dst_page, dst_slot = table[b, to // page], to % page
    stays = ((k < a) & (path == k)).sum(1, keepdim=True)        # the path's first nodes, which keep their places
    span = (L // page + torch.arange(6, device=DEV)[None]).clamp(max=s["width"] - 1)
    near = table.gather(1, span)                                # pages that drafts lie on
    kept = (span * page)[..., None] + torch.arange(page, device=DEV) < (L + stays)[..., None]
    after = []
    for n, cache in enumerate((s["k"], s["v"])):
        before, bits = s["exp"][..., n].int(), cache.view(torch.uint8)
        rows = cache.view(torch.uint8)[src_page, :, src_slot].view(torch.float8_e4m3fn).float() * _two(before[src_page])[..., None]
        e = before.scatter_reduce(0, dst_page[:, None].expand(-1, hkv), _need(_magnitude(rows)), "amax")
        up = (e - before)[near][..., None, None]
        was = bits[near]
        again = _encode(was.view(torch.float8_e4m3fn).float(), up.clamp(min=0))
        bits[near] = torch.where(kept[:, :, None, :, None] & (up > 0), again.view(torch.uint8), was)
        bits[dst_page, :, dst_slot] = _encode(rows, e[dst_page][..., None]).view(torch.uint8)
        after.append(e)
    s["exp"].copy_(torch.stack(after, -1))
    lens += s["accepted"]
    return [s["k"], s["v"], s["exp"], lens]


def _scored_rows(s):
    """The packed row under which each drafted token is scored: its parent's."""
    n = s["logits"].shape[0]
    at = torch.arange(n, device=DEV)
    off = s["offsets"].long()
    seq = torch.searchsorted(off, at, right=True) - 1
    return off[seq] + s["parent"].long().clamp(min=0), s["parent"] < 0


def _score(s, dtype):
    top = s["case"]["top"]
    x = s["logits"].to(dtype)
    m = x.amax(1, keepdim=True)
    w = (x - m).exp()
    total = w.sum(1, keepdim=True)
    lse = m + total.log()
    entropy = total.log()[:, 0] - (w * (x - m)).sum(1) / total[:, 0]
    row, root = _scored_rows(s)
    logprob = torch.where(root, 0.0, x[row, s["tokens"].long()] - lse[row, 0])
    v, ids = torch.sort(x, dim=1, descending=True, stable=True) if top else (x, x)
    return logprob, entropy, lse[:, 0], ids[:, :top].int(), v[:, :top] - lse


def _run_logprobs(s):
    o = s["out"]
    if own:
        s["ctx"].owl_token_logprobs(s["dims"], s["logits"], s["tokens"], s["offsets"], s["parent"], o["logprob"], o["entropy"], o["lse"], o["top_ids"],
                                    o["top_logprobs"])
        return o
    return dict(zip(("logprob", "entropy", "lse", "top_ids", "top_logprobs"), _score(s, torch.float32)))


# ------------------------------------------------------------------------------------------------------------ in 64 bits
def _exact_logprobs(s):
    c = s["case"]
    x = s["logits"].double()
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse[:, None])
    entropy = -(p * (x - lse[:, None])).sum(1)
    parent, tokens = s["parent"].cpu().numpy(), s["tokens"].cpu().numpy()
    first = (np.arange(len(parent)) // c["nodes"]) * c["nodes"]
    row = torch.as_tensor(np.where(parent < 0, 0, first + parent), device=DEV)
    logprob = x[row, torch.as_tensor(tokens, device=DEV).long()] - lse[row]
    logprob[torch.as_tensor(parent < 0, device=DEV)] = 0.0
    best = torch.topk(x, c["top"], 1).values if c["top"] else x[:, :0]
    return {"logprob": logprob, "entropy": entropy, "lse": lse, "top_ids": None, "top_logprobs": best - lse[:, None]}


def _exact_append(s):
    c = s["case"]
    hq, hkv, page = c["hq"], c["hkv"], c["page"]
    x = s["qkv"].double()
    row = s["rope"].double()[s["positions"].long()]
    w = torch.complex(row[:, :64], row[:, 64:])[:, None]
    turned = torch.complex(x[:, :hq + hkv, :64], x[:, :hq + hkv, 64:]) * w
    turned = torch.cat([turned.real, turned.imag], -1)
    q, k, v = turned[:, :hq], turned[:, hq:], x[:, hq + hkv:]
    if c["cache"] == "8":
        return [q, None, None, None]
    table, lens, off = s["table"].cpu().numpy(), s["lens"].cpu().numpy(), s["offsets"].cpu().numpy()
    outs = []
    for cache, new in ((s["k"], k), (s["v"], v)):
        flat = cache.double()
        for b in range(c["batch"]):
            pos = np.arange(lens[b], lens[b] + off[b + 1] - off[b])
            pg = torch.as_tensor(table[b, pos // page].astype(np.int64), device=DEV)
            flat[pg, :, torch.as_tensor(pos % page, device=DEV)] = new[off[b]:off[b + 1]]
        outs.append(flat)
    return [q] + outs


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "logprobs":
        return _exact_logprobs(s)
    if case["op"] == "append":
        return _exact_append(s)
    if case["op"] == "commit":
        return None                # bytes and whole exponents: nothing computed in between
    return _exact_attention(s)


def _exact_attention(s):
    c = s["case"]
    g = c["hq"] // c["hkv"]
    table, lens, off, parent = (s[k].cpu().numpy() for k in ("table", "lens", "offsets", "parent"))
    out = torch.zeros((s["total"], c["hq"], D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["total"], c["hq"]), dtype=torch.float64, device=DEV)
    for b in range(c["batch"]):
        L, n = int(lens[b]), int(off[b + 1] - off[b])
        sees = np.zeros((n, L + n), dtype=bool)
        sees[:, :L] = True
        for i in range(n):
            j = i
            while j >= 0:
                sees[i, L + j] = True
                j = int(parent[off[b] + j])
        sees = torch.as_tensor(sees, device=DEV)
        pages = torch.as_tensor(table[b, :(L + n + c["page"] - 1) // c["page"]].astype(np.int64), device=DEV)
        for h in range(c["hkv"]):
            kv = []
            for i, cache in enumerate((s["k"], s["v"])):
                x = cache.view(torch.uint8)[pages, h].view(torch.float8_e4m3fn).double() * torch.exp2(s["exp"][pages, h, i].double())[:, None, None]
                kv.append(x.reshape(-1, D)[:L + n])
            q = s["q"][off[b]:off[b + 1], h * g:(h + 1) * g].double()
            x = torch.einsum("igd,kd->igk", q, kv[0]) * s["scale"]
            x = torch.where(sees[:, None, :], x, -math.inf)
            z = torch.logsumexp(x, -1)
            out[off[b]:off[b + 1], h * g:(h + 1) * g] = torch.einsum("igk,kd->igd", torch.exp(x - z[..., None]), kv[1])
            lse[off[b]:off[b + 1], h * g:(h + 1) * g] = z
    return [out, lse]
