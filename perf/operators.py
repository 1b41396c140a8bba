"""Measured cases of the 4-bit target cache: what a drafting server calls to extend, fill, read and attend it.

Four kinds of case, each one pass of a public entry point:
  extend  page tables and slot maps of the newly verified tokens, from the lengths and the list of free pages
  store   K and V of new tokens quantised into the cache's slots, and read back as the values the slots now hold
  load    the values of given slots
  attn    draft attention over [4-bit target cache | draft K/V], with an optional sliding window and sink tokens
Sizes are those of the benchmark's workloads, of the parity tests, or generic.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 128
BLOCK = 16          # dims that share a scale
GROUP = 16          # tokens of a group of the cache's layout
GROUP_BYTES = 2304  # 16 tokens x (K codes 64 B, V codes 64 B, K scales 8 B, V scales 8 B)


def _extend(name, caches, min_len, max_len, min_new, max_new, page, lens_seed=0):
    case = {"kind": "extend", "caches": caches, "min_len": min_len, "max_len": max_len, "min_new": min_new,
            "max_new": max_new, "page": page, "lens_seed": lens_seed}
    return {"name": name, **case} if name else case


def _rows(name, kind, tokens, hkv=8, page=16, fused=0, run=1, k_exp=0, v_exp=0):
    """fused: query heads of the fused projection whose rows K and V are slices of (0: K and V are tensors of their own);
    run: consecutive tokens of a cache that stand together."""
    case = {"kind": kind, "tokens": tokens, "hkv": hkv, "page": page, "fused": fused, "run": run, "k_exp": k_exp,
            "v_exp": v_exp}
    return {"name": name, **case} if name else case


def _attn(name, *, seqs=1, layers=1, min_len, max_len, nodes, query, width=0, hq=32, hkv=8, page=16, window=0, sinks=0,
          k_exp=0, v_exp=0, lens_seed=0):
    """width: nodes of a level of the draft tree (0: a chain); page 0: a contiguous cache."""
    case = {"kind": "attn", "seqs": seqs, "layers": layers, "min_len": min_len, "max_len": max_len, "nodes": nodes,
            "query": query, "width": width, "hq": hq, "hkv": hkv, "page": page, "window": window, "sinks": sinks,
            "k_exp": k_exp, "v_exp": v_exp, "lens_seed": lens_seed}
    return {"name": name, **case} if name else case


def listed():
    return [
        # between two verification steps of a serving batch: each sequence has accepted one to eight tokens
        _extend("extend-64-decode", 64, 512, 8192, 1, 8, 16, lens_seed=4),
        # a batch of new prompts, none of which has a page yet
        _extend("extend-256-prompts", 256, 0, 0, 1, 8191, 16, lens_seed=5),
        # one verified token of each of 64 sequences, K and V as slices of the fused projection's rows
        _rows("store-64", "store", 64, fused=32),
        # the chunk of a long prompt
        _rows("store-32k", "store", 32771, page=64, run=32771),
        # a short prefix read back
        _rows("load-2k", "load", 2048, run=2048),
        # the ragged prefixes of a batch, page by page
        _rows("load-128k", "load", 131009, run=512),
        # one conversation, one drafted token at a time: a call of a few microseconds
        _attn("attn-1x2k", min_len=2048, max_len=2048, nodes=8, query=1, page=0),
        # a serving batch of mixed lengths, chain drafting
        _attn("attn-ragged-64", seqs=64, min_len=512, max_len=8192, nodes=8, query=1, lens_seed=4, v_exp=-1),
        # the fullest level of a batched draft tree
        _attn("attn-16x4k-level", seqs=16, min_len=4096, max_len=4096, nodes=56, query=12, width=12),
        # the same tree in one call (256 query rows per KV head): compute weighs more than bandwidth
        _attn("attn-16x4k-whole", seqs=16, min_len=4096, max_len=4096, nodes=64, query=64, width=12),
        # long contexts, four reused target layers attended separately: the largest working set
        _attn("attn-4x4x32k", seqs=4, layers=4, min_len=32768, max_len=32768, nodes=32, query=4, width=4, page=64),
        # long contexts of a target that attends to a window and the first tokens only
        _attn("attn-16x32k-window", seqs=16, min_len=20011, max_len=32768, nodes=8, query=1, page=64, window=4096,
              sinks=16, lens_seed=7),
    ]


MAX_KEYS = 16 * 32768 * 8   # keys x KV heads of the largest listed case
MAX_PAIRS = MAX_KEYS * 16   # and its (row, key) pairs


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["extend"] * 2 + ["store"] * 2 + ["load"] * 2 + ["attn"] * 6)
    if kind == "extend":
        caches, page = _log_int(rng, 1, 1024), rng.choice([16, 32, 64, 128])
        seed = rng.randrange(1 << 20)
        if rng.random() < 0.5:
            most = _log_int(rng, 64, 16384)
            return _extend(None, caches, most // 16, most, 0, rng.randint(1, 9), page, seed)
        return _extend(None, caches, 0, 0, 0, _log_int(rng, 2, max(3, (1 << 20) // caches)), page, seed)
    if kind in ("store", "load"):
        hkv = rng.choice([1, 2, 4, 8, 8, 8])
        tokens = _log_int(rng, 1, 32768 if kind == "store" else 131072)
        run_ = rng.choice([1, tokens, rng.randint(2, 600)])
        run_ = min(tokens, max(run_, -(-tokens // 512)))  # up to 512 caches
        return _rows(None, kind, tokens, hkv, rng.choice([16, 32, 64, 128, 256]),
                     rng.choice([0, 4 * hkv]) if kind == "store" else 0, run_, rng.choice([0, 0, -3, 2]),
                     rng.choice([0, 0, -3, 2]))
    hq, hkv = rng.choice([(32, 8), (32, 8), (32, 8), (32, 4), (16, 8), (64, 8), (8, 8), (28, 4)])
    seqs, layers = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 3, 4])
    width = rng.choice([0, 0, 1, 4, 8, 12])
    nodes = rng.randint(1, 64) if width else _log_int(rng, 1, 100)
    query = min(nodes, rng.choice([1, 1, 1, max(1, width), max(1, width), rng.randint(1, nodes), nodes]))
    rows = query * (hq // hkv)
    budget = min(MAX_KEYS, MAX_PAIRS // max(16, rows))
    max_len = _log_int(rng, 1, min(32768, max(65, budget // (seqs * layers * hkv))))
    min_len = max_len if rng.random() < 0.4 else max_len // rng.choice([2, 4, 16])
    window = rng.choice([0, 0, 0, rng.randint(1, 64), _log_int(rng, 16, 8192)])
    return _attn(None, seqs=seqs, layers=layers, min_len=min_len, max_len=max_len, nodes=nodes, query=query,
                 width=width, hq=hq, hkv=hkv, page=rng.choice([0, 16, 16, 32, 64, 128, 256]), window=window,
                 sinks=rng.choice([0, 4, 16, rng.randint(1, 200)]) if window else 0, k_exp=rng.choice([0, 0, -2, 3]),
                 v_exp=rng.choice([0, 0, -2, 3]), lens_seed=rng.randrange(1 << 20))


# ------------------------------------------------------------------ inputs

def _lens(case, lo="min_len", hi="max_len", n=None, salt=0):
    n = n or case.get("caches") or case["seqs"] * case["layers"]
    return np.random.default_rng(case["lens_seed"] + salt).integers(case[lo], case[hi], size=n, endpoint=True)


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(shape, g, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)


def _keys(shape, g):
    """Keys: a few channels are several times the others, as target keys have them."""
    channel = torch.exp(0.7 * torch.randn(shape[-1], generator=g, device="cuda"))
    return (torch.randn(shape, generator=g, device="cuda") * channel * 0.7).to(torch.bfloat16)


def _quantise(x, exp):
    """Codes [..., 128] (e2m1: sign, 2 exponent bits, 1 mantissa bit) and scales [..., 8] (e4m3) of x."""
    b = x.float().reshape(*x.shape[:-1], D // BLOCK, BLOCK)
    top = b.abs().amax(-1) * 2.0 ** -exp
    # (a tensor's division: by a number it would be a product with a rounded 1/6, which misses ties)
    s = (top / torch.full_like(top, 6.0)).clamp(2.0 ** -9, 448.0).to(torch.float8_e4m3fn)
    a, t = b.abs(), (s.float() * 2.0 ** exp)[..., None]
    # midpoints of 0, .5, 1, 1.5, 2, 3, 4, 6, ties to the even code; their products with a scale are exact
    code = ((a > t * 0.25).to(torch.uint8) + (a >= t * 0.75) + (a > t * 1.25) + (a >= t * 1.75) + (a > t * 2.5)
            + (a >= t * 3.5) + (a > t * 5.0))
    return (code + 8 * torch.signbit(b)).to(torch.uint8).reshape(x.shape), s


def _values(code, s, exp):
    """What codes and scales stand for, in 32 bits."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    v = table[code.int()].reshape(*code.shape[:-1], D // BLOCK, BLOCK)
    return (v * (s.float() * 2.0 ** exp)[..., None]).reshape(code.shape)


def _pack(kc, ks, vc, vs):
    """Codes and scales of groups [G, 16 tokens, ...] in the cache's layout: chunks of 32 dims, 16 tokens to a chunk."""
    def codes(c):
        byte = c[..., 0::2] | (c[..., 1::2] << 4)
        return byte.reshape(-1, GROUP, 4, 16).transpose(1, 2).reshape(-1, 1024)
    scales = [s.view(torch.uint8).reshape(-1, 128) for s in (ks, vs)]
    return torch.cat([codes(kc), codes(vc), *scales], dim=1)


def _unpack(groups):
    """[..., 2304] bytes -> codes [..., 16, 128] and scales [..., 16, 8] of K and of V."""
    def codes(b):
        b = b.reshape(*b.shape[:-1], 4, GROUP, 16).transpose(-3, -2).reshape(*b.shape[:-1], GROUP, 64)
        return torch.stack([b & 15, b >> 4], dim=-1).reshape(*b.shape[:-1], D)
    def scales(b):  # noqa: E306
        return b.contiguous().view(torch.float8_e4m3fn).reshape(*b.shape[:-1], GROUP, 8)
    return (codes(groups[..., :1024]), scales(groups[..., 2048:2176]), codes(groups[..., 1024:2048]),
            scales(groups[..., 2176:]))


def _random_cache(pages, hkv, page, g, k_exp, v_exp):
    """A filled cache [pages, hkv, page / 16, 2304] of quantised keys and values."""
    n = pages * hkv * (page // GROUP)
    out = torch.empty((n, GROUP_BYTES), dtype=torch.uint8, device="cuda")
    step = 1 << 14
    for i in range(0, n, step):
        m = min(step, n - i)
        kc, ks = _quantise(_keys((m, GROUP, D), g), k_exp)
        vc, vs = _quantise(_randn((m, GROUP, D), g), v_exp)
        out[i:i + m] = _pack(kc, ks, vc, vs)
    return out.reshape(pages, hkv, page // GROUP, GROUP_BYTES)


def _int(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def prepare(case, seed):
    g, rng = _generator(seed), np.random.default_rng(seed)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    st = {"case": case, "err": err}
    page = case["page"]
    if case["kind"] == "extend":
        lens, new = _lens(case), _lens(case, "min_new", "max_new", salt=1)
        c, used = len(lens), -(-lens // page)
        per = int((-(-(lens + new) // page)).max()) + 1
        need = int((-(-(lens + new) // page) - used).sum())
        ids = rng.permutation(int(used.sum()) + need + 37)
        table = np.zeros((c, per), np.int32)
        held = np.arange(per)[None, :] < used[:, None]
        table[held] = ids[:held.sum()]
        free = ids[held.sum():]
        total = int(new.sum()) + 5
        st |= {"lens": _int(lens), "new": _int(new), "table": _int(table), "free": _int(free),
               "count": _int([len(free)]), "pages": len(ids), "total": total}
        if own:  # the outputs' buffers and the descriptor, which a program keeps
            from paper_2604_26412_gb300 import kvshot
            empty = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")  # noqa: E731
            st["out"] = {"lens": empty(c), "table": empty(c, per), "count": empty(1), "start": empty(c + 1),
                         "slots": empty(total), "cache": empty(total), "pos": empty(total)}
            st["desc"] = kvshot.make_extend_desc(num_caches=c, page_size=page, max_pages_per_seq=per,
                                                 num_pages=len(ids), max_tokens=total, err_flag=err)
        return st
    if case["kind"] in ("store", "load"):
        t, hkv, run_ = case["tokens"], case["hkv"], case["run"]
        # runs of consecutive tokens, each in pages of its own, every run at a random place of its first page
        runs, span = -(-t // run_), -(-run_ // page) + 1
        pages = runs * span
        first = rng.integers(0, page, size=runs)
        ids = rng.permutation(pages).reshape(runs, span)
        i = np.arange(t)
        at = first[i // run_] + i % run_
        st["slots"] = _int(ids[i // run_, at // page] * page + at % page)
        if case["kind"] == "store":
            heads = case["fused"] + 2 * hkv
            qkv = _randn((t, heads, D), g)
            k, v = qkv[:, heads - 2 * hkv:heads - hkv], qkv[:, heads - hkv:]
            k.copy_(_keys(k.shape, g))
            st |= {"k": k, "v": v} if case["fused"] else {"k": k.contiguous(), "v": v.contiguous()}
            st["cache"] = torch.zeros((pages, hkv, page // GROUP, GROUP_BYTES), dtype=torch.uint8, device="cuda")
        else:
            st["cache"] = _random_cache(pages, hkv, page, g, case["k_exp"], case["v_exp"])
        if own:
            from paper_2604_26412_gb300 import kvshot
            st["out"] = {n: torch.empty((t, hkv, D), dtype=torch.bfloat16, device="cuda") for n in ("k", "v")}
            stride = st["k"].stride(0) if case["kind"] == "store" else 0
            sizes = dict(num_tokens=t, hkv=hkv, page_size=page, num_pages=pages, k_scale_exp=case["k_exp"],
                         v_scale_exp=case["v_exp"], err_flag=err)
            st["desc"] = kvshot.make_kv4_desc(**sizes, k_stride=stride, v_stride=stride)
            st["back"] = kvshot.make_kv4_desc(**sizes)
        return st
    c, hq, hkv, n, nq = case["seqs"] * case["layers"], case["hq"], case["hkv"], case["nodes"], case["query"]
    lens = _lens(case)
    per = -(-max(1, int(lens.max())) // (page or GROUP))
    if page:
        used = -(-lens // page)
        table = np.zeros((c, per), np.int64)
        held = np.arange(per)[None, :] < used[:, None]
        table[held] = rng.permutation(int(used.sum()))
        st["table"], pages = _int(table), max(1, int(used.sum()))
    else:
        st["table"], pages = None, c
    st["page"] = page or per * GROUP  # a contiguous cache is one page per cache
    st["cache"] = _random_cache(pages, hkv, st["page"], g, case["k_exp"], case["v_exp"])
    st["lens"] = _int(lens)
    st["parent"] = None
    if case["width"]:
        w = case["width"]
        i = np.arange(n)
        st["parent"] = _int(np.where(i < w, -1, (i // w - 1) * w + rng.integers(0, w, size=(case["seqs"], n))))
    st["q"] = _randn((c, nq, hq, D), g)
    slots = -(-n // 8) * 8
    st["draft_k"], st["draft_v"] = _keys((c, hkv, slots, D), g), _randn((c, hkv, slots, D), g)
    if own:
        from paper_2604_26412_gb300 import kvshot
        st["out"] = {"out": torch.empty_like(st["q"]), "lse": torch.empty((c, nq, hq), device="cuda")}
        st["desc"] = kvshot.make_desc(
            num_caches=c, num_seqs=case["seqs"], hq=hq, hkv=hkv, n_nodes=n, n_query=nq, n_max=slots,
            max_seq_len=int(lens.max()), page_size=page, max_pages_per_seq=per if page else 0,
            num_pages=pages if page else 0, l_cap=0 if page else st["page"], tree=case["width"] > 0, err_flag=err,
            k_scale_exp=case["k_exp"], v_scale_exp=case["v_exp"])
        size = kvshot.draft_attn_kv4_workspace_size(st["desc"], case["window"], case["sinks"])
        st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        st["desc"].workspace, st["desc"].workspace_bytes = st["workspace"].data_ptr(), size
    return st


# ------------------------------------------------------------------ one pass

def _plain_extend(st):
    page, lens, new = st["case"]["page"], st["lens"], st["new"]
    used, after = (lens + page - 1) // page, (lens + new + page - 1) // page
    need = after - used
    base = torch.cumsum(need, 0) - need
    col = torch.arange(st["table"].shape[1], device="cuda")
    fresh = (col >= used[:, None]) & (col < after[:, None])
    at = st["count"] - 1 - (base[:, None] + col - used[:, None])
    table = torch.where(fresh, st["free"][at.clamp(0, st["free"].numel() - 1).long()], st["table"])
    start = torch.cat([torch.zeros_like(lens[:1]), torch.cumsum(new, 0)]).int()
    t = torch.arange(st["total"], device="cuda", dtype=torch.int32)
    cache = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp(max=lens.numel() - 1)
    pos = lens[cache] + t - start[cache]
    slots = table[cache, (pos // page).clamp(max=table.shape[1] - 1).long()] * page + pos % page
    live = t < start[-1]
    none = torch.full_like(t, -1)
    return {"lens": lens + new, "table": table, "count": (st["count"] - need.sum()).int(), "start": start,
            "slots": torch.where(live, slots.int(), none), "cache": torch.where(live, cache.int(), none),
            "pos": torch.where(live, pos.int(), none)}


def _plain_load(st):
    case, page = st["case"], st["case"]["page"]
    slot = st["slots"].long()
    group = st["cache"][slot // page, :, slot % page // GROUP]  # [T, hkv, 2304]
    t = torch.arange(slot.numel(), device="cuda")
    row = slot % GROUP
    kc, ks, vc, vs = (x[t, :, row] for x in _unpack(group))
    return {"k": _values(kc, ks, case["k_exp"]).to(torch.bfloat16), "v": _values(vc, vs, case["v_exp"]).to(torch.bfloat16)}


def _plain_attn(st):
    case = st["case"]
    c, hq, hkv, n, nq = case["seqs"] * case["layers"], case["hq"], case["hkv"], case["nodes"], case["query"]
    g, page = hq // hkv, st["page"]
    length = st["lens"].long()
    table = st["table"].long() if st["table"] is not None else torch.arange(c, device="cuda")[:, None]
    groups = st["cache"][table].transpose(1, 2)  # [C, hkv, pages, groups, 2304]
    kc, ks, vc, vs = (x.reshape(c, hkv, -1, x.shape[-1]) for x in _unpack(groups))
    m = kc.shape[2]
    k = torch.cat([_values(kc, ks, case["k_exp"]), st["draft_k"][:, :, :n].float()], dim=2)
    v = torch.cat([_values(vc, vs, case["v_exp"]), st["draft_v"][:, :, :n].float()], dim=2)
    del kc, ks, vc, vs, groups
    # ancestors of every node, itself among them, and positions: a node stands at L + depth - 1
    i = torch.arange(n, device="cuda")
    parent = st["parent"].long() if st["parent"] is not None else (i - 1)[None, :].expand(case["seqs"], n)
    step = (parent[:, :, None] == i).double() + torch.eye(n, dtype=torch.float64, device="cuda")
    see = torch.linalg.matrix_power(step, n) > 0
    depth = see.sum(-1)
    see, depth = see.repeat_interleave(case["layers"], 0), depth.repeat_interleave(case["layers"], 0)
    pos = length[:, None] + depth - 1                                                  # [C, n]
    at = torch.cat([torch.arange(m, device="cuda").expand(c, m), pos], dim=1)          # of every key
    row = pos[:, n - nq:]
    mask = torch.cat([(torch.arange(m, device="cuda") < length[:, None])[:, None].expand(c, nq, m), see[:, n - nq:]], 2)
    if case["window"]:
        mask = mask & ((row[:, :, None] - at[:, None] < case["window"]) | (at < case["sinks"])[:, None])
    q = st["q"].float().reshape(c, nq, hkv, g, D).permute(0, 2, 1, 3, 4).reshape(c, hkv, nq * g, D)
    s = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    s = s.masked_fill(~mask.repeat_interleave(g, 1)[:, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / z
    lse = (top + torch.log(z)).reshape(c, hkv, nq, g).permute(0, 2, 1, 3).reshape(c, nq, hq)
    return {"out": o.reshape(c, hkv, nq, g, D).permute(0, 2, 1, 3, 4).reshape(c, nq, hq, D).to(torch.bfloat16),
            "lse": lse}


def run(state):
    st, case = state, state["case"]
    if own:
        from paper_2604_26412_gb300 import kvshot
        o = st["out"]
        if case["kind"] == "extend":
            kvshot.cache_extend(st["desc"], st["lens"], st["new"], st["table"], st["free"], st["count"], o["lens"],
                                o["table"], o["count"], o["start"], o["slots"], o["cache"], o["pos"])
        elif case["kind"] == "attn":
            kvshot.draft_attn_kv4(st["desc"], st["q"], st["cache"], st["table"], st["lens"], st["draft_k"],
                                  st["draft_v"], st["parent"], case["window"], case["sinks"], o["out"], o["lse"])
        else:
            if case["kind"] == "store":
                kvshot.kv4_store(st["desc"], st["k"], st["v"], st["slots"], st["cache"])
            kvshot.kv4_load(st["back"], st["cache"], st["slots"], o["k"], o["v"])
        return {**o, "err": st["err"]}
    if case["kind"] == "extend":
        o = _plain_extend(st)
    elif case["kind"] == "store":
        o = {x: _values(*_quantise(st[x], case[x + "_exp"]), case[x + "_exp"]).to(torch.bfloat16) for x in ("k", "v")}
    elif case["kind"] == "load":
        o = _plain_load(st)
    else:
        o = _plain_attn(st)
    return {**o, "err": st["err"]}


def _visible(case):
    """Prefix keys of each cache that some query row sees, by the shallowest row's window."""
    lens = _lens(case)
    if not case["window"]:
        return lens
    n, nq, w = case["nodes"], case["query"], case["width"]
    depth = (n - nq) // w if w else n - nq  # of the first query row, less one
    first = np.maximum(0, lens + depth - case["window"] + 1)
    return np.minimum(lens, np.minimum(case["sinks"], first) + np.maximum(0, lens - first))


def work(case):
    if case["kind"] == "extend":
        lens, new = _lens(case), _lens(case, "min_new", "max_new", salt=1)
        after = -(-(lens + new) // case["page"])
        c, t, per = len(lens), int(new.sum()) + 5, int(after.max()) + 1
        need = int((after - -(-lens // case["page"])).sum())
        return {"bytes": 4 * (2 * c + c * per + need + c + c * per + c + 1 + 3 * t), "flops": 0}
    if case["kind"] in ("store", "load"):
        t, hkv = case["tokens"], case["hkv"]
        passes = 2 if case["kind"] == "store" else 1  # stored, then read back
        return {"bytes": passes * t * (hkv * (4 * D + 144) + 4), "flops": 0}
    c, hq, hkv, n, nq = case["seqs"] * case["layers"], case["hq"], case["hkv"], case["nodes"], case["query"]
    seen = int(_visible(case).sum())
    total = seen * hkv * 144 + c * n * hkv * D * 4 + c * nq * hq * (4 * D + 4) + 4 * c
    total += 4 * -(-seen // case["page"]) if case["page"] else 0
    total += 4 * case["seqs"] * n if case["width"] else 0
    return {"bytes": total, "flops": 4 * D * hq * nq * (seen + c * n)}


# ------------------------------------------------------------------ the same in 64 bits

def _e4m3(b):
    """The values of e4m3 bytes, from the format: sign, 4 exponent bits of bias 7, 3 mantissa bits."""
    b = b.to(torch.int64)
    e, m = (b >> 3) & 15, (b & 7).double()
    power = torch.tensor([2.0 ** (i - 7) for i in range(16)], dtype=torch.float64, device=b.device)  # exact
    v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * power[e])
    return torch.where(b >= 128, -v, v)


def _slot_values(cache, page, pages_of, offset, head, exp, kind):
    """K (kind 0) or V (kind 1) of the tokens at (page, offset) for one head, from the layout byte by byte."""
    group, row = offset // GROUP, offset % GROUP
    flat = cache[pages_of, head, group]
    d = torch.arange(D, device=cache.device)
    byte = flat.gather(1, kind * 1024 + (d // 32)[None] * 256 + row[:, None] * 16 + (d % 32 // 2)[None])
    nib = (byte.to(torch.int64) >> (4 * (d % 2))[None]) & 15
    e, m, neg = (nib >> 1) & 3, (nib & 1).double(), nib >= 8
    power = torch.tensor([0.5, 1.0, 2.0, 4.0], dtype=torch.float64, device=cache.device)
    mag = torch.where(e == 0, m / 2, (1 + m / 2) * power[e])
    scale = _e4m3(flat.gather(1, 2048 + kind * 128 + row[:, None] * 8 + (d // BLOCK)[None]))
    return torch.where(neg, -mag, mag) * scale * 2.0 ** exp


def _nearest(x, grid):
    """Index of the nearest of the ascending values `grid`, ties to the even one, saturating."""
    i = torch.searchsorted(grid, x.contiguous()).clamp(1, grid.numel() - 1)
    lo, hi = grid[i - 1], grid[i]
    up = (x - lo > hi - x) | ((x - lo == hi - x) & (i % 2 == 0))
    return torch.where(up, i, i - 1)


def _exact_store(x, exp):
    e4m3 = _e4m3(torch.arange(0x7F, device=x.device))
    e2m1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    out = []
    for part in torch.split(x, 4096):
        b = part.double().reshape(*part.shape[:-1], D // BLOCK, BLOCK)
        top = b.abs().amax(-1) * 2.0 ** -exp
        s = e4m3[_nearest(top, 6 * e4m3).clamp(min=1)][..., None] * 2.0 ** exp  # 6 times a scale is exact
        out.append((e2m1[_nearest(b.abs() / s, e2m1)] * s * torch.sign(b)).reshape(part.shape))
    return torch.cat(out)


def _exact_extend(st):
    page, lens, new = st["case"]["page"], st["lens"].cpu().numpy(), st["new"].cpu().numpy()
    table, free = st["table"].cpu().numpy().copy(), st["free"].cpu().numpy().tolist()
    start, slots, cache, pos = [0], [], [], []
    for c in range(len(lens)):
        for p in range(-(-int(lens[c]) // page), -(-int(lens[c] + new[c]) // page)):
            table[c, p] = free.pop()
        at = lens[c] + np.arange(new[c])
        slots.append(table[c, at // page] * page + at % page)
        cache.append(np.full(new[c], c))
        pos.append(at)
        start.append(start[-1] + int(new[c]))
    pad = [np.full(st["total"] - start[-1], -1)]
    whole = lambda x: np.asarray(np.concatenate(x + pad), dtype=np.int32)  # noqa: E731
    return {"lens": lens + new, "table": table, "count": np.array([len(free)], np.int32),
            "start": np.array(start, np.int32), "slots": whole(slots), "cache": whole(cache), "pos": whole(pos),
            "err": None}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "extend":
        return _exact_extend(st)
    if case["kind"] == "store":
        return {"k": _exact_store(st["k"], case["k_exp"]), "v": _exact_store(st["v"], case["v_exp"]), "err": None}
    if case["kind"] == "load":
        slot = st["slots"].long()
        per_head = lambda kind, e: torch.stack([_slot_values(st["cache"], case["page"], slot // case["page"], slot % case["page"], h, e, kind)  # noqa: E731
                                                for h in range(case["hkv"])], dim=1)
        return {"k": per_head(0, case["k_exp"]), "v": per_head(1, case["v_exp"]), "err": None}
    c_, hq, hkv, n, nq = case["seqs"] * case["layers"], case["hq"], case["hkv"], case["nodes"], case["query"]
    g, page = hq // hkv, st["page"]
    out = torch.empty((c_, nq, hq, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((c_, nq, hq), dtype=torch.float64, device="cuda")
    parent = st["parent"].cpu().numpy() if st["parent"] is not None else None
    for c in range(c_):
        length = int(st["lens"][c])
        line = []  # of each node: the nodes from it to its root
        for i in range(n):
            up = (int(parent[c // case["layers"], i]) if parent is not None else i - 1)
            line.append([i] + (line[up] if up >= 0 else []))
        at = [length + len(x) - 1 for x in line]
        mask = torch.zeros((nq, length + n), dtype=torch.bool)
        for r, i in enumerate(range(n - nq, n)):
            j = torch.arange(length)
            mask[r, :length] = True if not case["window"] else (at[i] - j < case["window"]) | (j < case["sinks"])
            for a in line[i]:
                mask[r, length + a] = not case["window"] or at[i] - at[a] < case["window"] or at[a] < case["sinks"]
        mask = mask.cuda().repeat_interleave(g, 0)
        j = torch.arange(length, device="cuda")
        pid = st["table"][c].long()[j // page] if st["table"] is not None else torch.full_like(j, c)
        for h in range(hkv):
            k = torch.cat([_slot_values(st["cache"], page, pid, j % page, h, case["k_exp"], 0), st["draft_k"][c, h, :n].double()])
            v = torch.cat([_slot_values(st["cache"], page, pid, j % page, h, case["v_exp"], 1), st["draft_v"][c, h, :n].double()])
            q = st["q"][c, :, h * g:(h + 1) * g].double().reshape(nq * g, D)
            s = (q @ k.T / math.sqrt(D)).masked_fill(~mask, -math.inf)
            z = torch.logsumexp(s, dim=1)
            out[c, :, h * g:(h + 1) * g] = (torch.exp(s - z[:, None]) @ v).reshape(nq, g, D)
            lse[c, :, h * g:(h + 1) * g] = z.reshape(nq, g)
    return {"out": out, "lse": lse, "err": None}
