"""Measured cases of drafting over a part of a long target cache: what a server calls to look at few of its pages, or to
keep few of its tokens.

Six kinds of case, each one pass of a public entry point:
  bounds   least and greatest key of each page, for the pages that got tokens
  scores   of every page and query row, the greatest score that a key between those bounds can have
  select   the best pages of each query row, or the tokens of a cache to keep, by their scores
  sparse   draft attention over the pages that were selected for each query row and KV head, and the draft K/V
  weights  the softmax weight that each cached token got from the query rows, added to what it had
  evict    the kept tokens' K, V and weights moved to the front of a cache, its other pages given back
Sizes are those of the benchmark's workloads, of the parity tests, or generic.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 128


def _case(name, kind, **sizes):
    case = {"kind": kind, **sizes}
    return {"name": name, **case} if name else case


def _bounds(name, *, caches, min_len, max_len, new=0, hkv=8, page=16, lens_seed=0):
    """new: tokens that each cache got since its bounds were last computed (0: all of them)."""
    return _case(name, "bounds", caches=caches, min_len=min_len, max_len=max_len, new=new, hkv=hkv, page=page,
                 lens_seed=lens_seed)


def _scores(name, *, caches, min_len, max_len, query, hq=32, hkv=8, page=16, lens_seed=0):
    return _case(name, "scores", caches=caches, min_len=min_len, max_len=max_len, query=query, hq=hq, hkv=hkv, page=page,
                 lens_seed=lens_seed)


def _select(name, *, caches, per, min_len, max_len, unit, keep, first, last, lens_seed=0):
    """per: rows of scores of each cache; unit: tokens of an entry; entries kept at the front and at the back."""
    return _case(name, "select", caches=caches, per=per, min_len=min_len, max_len=max_len, unit=unit, keep=keep,
                 first=first, last=last, lens_seed=lens_seed)


def _sparse(name, *, seqs, layers=1, min_len, max_len, nodes, query, width=0, keep, hq=32, hkv=8, page=16, lens_seed=0):
    """width: nodes of a level of the draft tree (0: a chain); keep: pages of a query row and KV head."""
    return _case(name, "sparse", seqs=seqs, layers=layers, min_len=min_len, max_len=max_len, nodes=nodes, query=query,
                 width=width, keep=keep, hq=hq, hkv=hkv, page=page, lens_seed=lens_seed)


def _weights(name, *, caches, min_len, max_len, query, decay=1.0, hq=32, hkv=8, page=16, lens_seed=0):
    """page 0: a contiguous cache."""
    return _case(name, "weights", caches=caches, min_len=min_len, max_len=max_len, query=query, decay=decay, hq=hq,
                 hkv=hkv, page=page, lens_seed=lens_seed)


def _evict(name, *, caches, min_len, max_len, keep, hkv=8, page=16, lens_seed=0):
    return _case(name, "evict", caches=caches, min_len=min_len, max_len=max_len, keep=keep, hkv=hkv, page=page,
                 lens_seed=lens_seed)


def listed():
    return [
        # between two verification steps of a serving batch: the last one or two pages of every sequence changed
        _bounds("bounds-64-decode", caches=64, min_len=512, max_len=8192, new=8, lens_seed=4),
        # long prompts, just stored: every page
        _bounds("bounds-16x32k", caches=16, min_len=32768, max_len=32768, page=64),
        # one conversation, one drafted token at a time: a call of a few microseconds
        _scores("scores-1x8k", caches=1, min_len=8192, max_len=8192, query=1),
        # a level of a batched draft tree over long contexts
        _scores("scores-16x32k-level", caches=16, min_len=20011, max_len=32768, query=12, lens_seed=7),
        # the pages of each node and KV head of that level
        _select("select-pages", caches=16, per=96, min_len=20011, max_len=32768, unit=16, keep=128, first=1, last=4,
                lens_seed=7),
        # the tokens that each cache keeps: long rows, few of them
        _select("select-tokens", caches=16, per=1, min_len=20011, max_len=32768, unit=1, keep=4096, first=16, last=512,
                lens_seed=7),
        # one conversation, one drafted token, an eighth of its pages
        _sparse("sparse-1x8k", seqs=1, min_len=8192, max_len=8192, nodes=8, query=1, keep=64),
        # the level of the batched draft tree, 2048 tokens of each long context for each node and KV head
        _sparse("sparse-16x32k-level", seqs=16, min_len=20011, max_len=32768, nodes=56, query=12, width=12, keep=128,
                lens_seed=7),
        # weights of a drafted token over one contiguous cache
        _weights("weights-1x8k", caches=1, min_len=8192, max_len=8192, query=1, page=0),
        # a whole draft tree over long contexts (256 query rows per KV head): the largest amount of arithmetic
        _weights("weights-16x32k-whole", caches=16, min_len=20011, max_len=32768, query=64, decay=0.875, page=64,
                 lens_seed=7),
        # a serving batch of mixed lengths, kept to 512 tokens each
        _evict("evict-ragged-64", caches=64, min_len=512, max_len=8192, keep=512, lens_seed=4),
        # long contexts kept to an eighth
        _evict("evict-16x32k", caches=16, min_len=32768, max_len=32768, keep=4096, page=64),
    ]


MAX_KEYS = 16 * 32768 * 8   # keys x KV heads of the largest listed cases
MAX_LEN = 32768


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_lens(rng, caches, hkv, budget=MAX_KEYS):
    max_len = _log_int(rng, 1, max(2, min(MAX_LEN, budget // (caches * hkv))))
    return {"min_len": max_len if rng.random() < 0.3 else max_len // rng.choice([2, 4, 16]), "max_len": max_len,
            "lens_seed": rng.randrange(1 << 20)}


def draw(rng):
    kind = rng.choice(["bounds", "scores", "select", "sparse", "sparse", "weights", "weights", "evict"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (32, 8), (32, 4), (16, 8), (64, 8), (8, 8), (28, 4), (32, 2)])
    page = rng.choice([8, 16, 16, 32, 64, 128, 256])
    if kind == "bounds":
        caches = _log_int(rng, 1, 128)
        return _bounds(None, caches=caches, new=rng.choice([0, 0, 1, rng.randint(1, 300)]), hkv=hkv, page=page,
                       **_draw_lens(rng, caches, hkv))
    if kind == "scores":
        caches, query = _log_int(rng, 1, 64), rng.choice([1, 1, rng.randint(2, 16), rng.randint(2, 64)])
        # entries of the scores, and their products, within the largest listed case's
        budget = min(MAX_KEYS, MAX_KEYS * 12 * 4 // (query * (hq // hkv)) * page // 16)
        return _scores(None, caches=caches, query=query, hq=hq, hkv=hkv, page=page, **_draw_lens(rng, caches, hkv, budget))
    if kind == "select":
        caches, unit = _log_int(rng, 1, 128), rng.choice([1, 1, 8, 16, 64])
        per = 1 if unit == 1 else rng.choice([1, 8, hkv, 12 * hkv])
        lens = _draw_lens(rng, caches, per, 16 * 32768 * 6 * unit)
        lens["max_len"] = max(lens["max_len"], 200 * unit)  # (some choice is left, at least in the last cache)
        keep = _log_int(rng, 1, lens["max_len"] // unit - 100)
        first = min(keep - 1, rng.choice([0, 1, rng.randint(0, 20)]))
        return _select(None, caches=caches, per=per, unit=unit, keep=keep, first=first,
                       last=min(keep - 1 - first, rng.choice([0, 1, keep // 4, keep // 2])), **lens)
    if kind == "sparse":
        seqs, layers = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 4])
        seqs = max(1, seqs // layers)
        width = rng.choice([0, 0, 1, 4, 8, 12])
        nodes = rng.randint(1, 64) if width else _log_int(rng, 1, 100)
        query = min(nodes, rng.choice([1, 1, 1, max(1, width), max(1, width), rng.randint(1, nodes)]))
        lens = _draw_lens(rng, seqs * layers, hkv)
        most = max(1, 16 * 12 * 8 * 2048 // (seqs * layers * query * hkv * page))  # pages within the largest listed case's
        keep = _log_int(rng, 1, max(2, min(most, -(-lens["max_len"] // page) + 1)))
        return _sparse(None, seqs=seqs, layers=layers, nodes=nodes, query=query, width=width, keep=min(keep, most), hq=hq,
                       hkv=hkv, page=page, **lens)
    if kind == "weights":
        caches, query = _log_int(rng, 1, 64), rng.choice([1, 1, rng.randint(1, 16), rng.randint(1, 64)])
        rows = query * (hq // hkv)
        return _weights(None, caches=caches, query=query, decay=rng.choice([1.0, 0.0, 0.9375, rng.uniform(0.5, 1)]), hq=hq,
                        hkv=hkv, page=rng.choice([0, page, page]),
                        **_draw_lens(rng, caches, hkv, min(MAX_KEYS, MAX_KEYS * 256 // rows)))
    caches = _log_int(rng, 1, 64)
    lens = _draw_lens(rng, caches, hkv)
    return _evict(None, caches=caches, keep=_log_int(rng, 1, max(2, lens["max_len"])), hkv=hkv, page=page, **lens)


# ------------------------------------------------------------------ inputs

def _count(case):
    return case["caches"] if "caches" in case else case["seqs"] * case["layers"]


def _lens(case):
    lens = np.random.default_rng(case["lens_seed"]).integers(case["min_len"], case["max_len"], size=_count(case),
                                                             endpoint=True)
    lens[-1] = case["max_len"]
    return lens


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


def _int(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _table(lens, page, rng, per=None):
    """Page table [C, per] of a shuffled pool with three pages to spare, and the pool's size."""
    used = -(-lens // page)
    per = per or max(1, int(used.max()))
    ids = rng.permutation(int(used.sum()) + 3)
    table = np.zeros((len(lens), per), np.int32)
    table[np.arange(per)[None, :] < used[:, None]] = ids[:int(used.sum())]
    return table, ids


def _picks(case):
    """Pages of each query row and KV head [C, Nq, hkv, keep], ascending, -1 behind the last, and their numbers: the first
    page, the last two, and the best of scores that a cache's nodes largely agree on."""
    rng = np.random.default_rng(case["lens_seed"] + 1)
    lens, nq, hkv, keep, page = _lens(case), case["query"], case["hkv"], case["keep"], case["page"]
    out = np.full((len(lens), nq, hkv, keep), -1, np.int32)
    counts = np.zeros((len(lens), nq, hkv), np.int32)
    for c, n in enumerate(-(-lens // page)):
        m = min(int(n), keep)
        if m:
            s = rng.standard_normal((1, hkv, n)) + 0.5 * rng.standard_normal((nq, hkv, n))
            s[..., 0] += 100
            s[..., -2:] += 50
            out[c, :, :, :m] = np.sort(np.argpartition(-s, m - 1, axis=-1)[..., :m], axis=-1)
        counts[c] = m
    return out, counts


def _kept(case, salt=1):
    """Tokens that each cache keeps [C, keep], ascending, -1 behind the last, and their numbers: some of the first, a run
    at the end, and others."""
    rng = np.random.default_rng(case["lens_seed"] + salt)
    lens, keep = _lens(case), case["keep"]
    out, counts = np.full((len(lens), keep), -1, np.int32), np.minimum(lens, keep).astype(np.int32)
    for c, (n, m) in enumerate(zip(lens, counts)):
        s = rng.random(n)
        s[:4] += 1
        s[n - m // 8:] += 1
        out[c, :m] = np.sort(np.argsort(-s, kind="stable")[:m])
    return out, counts


def _gather(pool, table, page):
    """Rows [C, hkv, tokens, 128] of a paged pool in the tables' order."""
    x = pool[table.long()]                                      # [C, pages, hkv, P, 128]
    return x.transpose(1, 2).reshape(x.shape[0], x.shape[2], -1, D)


def _logsumexp(st, scale):
    """lse [C, Nq, hq] of the query rows over the whole prefix and one draft key of score 0."""
    case = st["case"]
    c_, hq, hkv, nq = case["caches"], case["hq"], case["hkv"], case["query"]
    lse = torch.empty((c_, nq, hq), device="cuda")
    for c in range(c_):
        k = _keys_of(st, c).float()                             # [hkv, L, 128]
        q = st["q"][c].float().reshape(nq, hkv, hq // hkv, D).permute(1, 0, 2, 3).reshape(hkv, -1, D)
        s = torch.matmul(q, k.transpose(1, 2)) * scale
        z = torch.logaddexp(torch.logsumexp(s, -1), torch.zeros((), device="cuda"))
        lse[c] = z.reshape(hkv, nq, hq // hkv).permute(1, 0, 2).reshape(nq, hq)
    return lse


def _keys_of(st, c):
    """Keys [hkv, L, 128] of cache c."""
    n, page = int(st["host_lens"][c]), st["case"]["page"]
    if not page:
        return st["k"][c, :, :n]
    used = max(1, -(-n // page))
    return _gather(st["k"], st["table"][c:c + 1, :used], page)[0, :, :n]


def prepare(case, seed):
    g, rng = _generator(seed), np.random.default_rng(seed)
    kind, lens = case["kind"], _lens(case)
    c, page = len(lens), case.get("page", 0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    st = {"case": case, "err": err, "lens": _int(lens), "host_lens": lens}
    if own:
        from paper_2604_26412_gb300 import kvshot
    if kind == "select":
        per, entries = case["per"], -(-lens // case["unit"])
        width = max(1, int(entries.max()))
        s = torch.randn((c * per, width), generator=g, device="cuda")
        if case["unit"] == 1:  # accumulated weights: many of them next to nothing, equal ones among them
            s = torch.exp(3 * s).to(torch.bfloat16).float()
        st["scores"] = s
        if own:
            st["out"] = {"picks": torch.empty((c * per, case["keep"]), dtype=torch.int32, device="cuda"),
                         "counts": torch.empty(c * per, dtype=torch.int32, device="cuda")}
            st["desc"] = kvshot.make_select_desc(
                num_rows=c * per, row_len=width, rows_per_len=per, tokens_per_entry=case["unit"], keep=case["keep"],
                first=case["first"], last=case["last"], err_flag=err)
        return st
    hkv = case["hkv"]
    if page:
        table, ids = _table(lens, page, rng)
        st["table"], pages = _int(table), len(ids)
    else:
        st["table"], pages = None, 0
        st["l_cap"] = max(1, int(lens.max()))
    attn = dict(num_caches=c, num_seqs=case.get("seqs", c), hq=case.get("hq", hkv), hkv=hkv, n_nodes=case.get("query", 0),
                n_query=case.get("query", 0), n_max=case.get("query", 0), max_seq_len=int(lens.max()), page_size=page,
                max_pages_per_seq=st["table"].shape[1] if page else 0, num_pages=pages, l_cap=st.get("l_cap", 0),
                err_flag=err)
    if kind == "bounds":
        st["k"] = _keys((pages, hkv, page, D), g)
        st["from"] = _int(np.maximum(0, lens - case["new"]) if case["new"] else np.zeros_like(lens))
        if own:
            st["out"] = {"bounds": torch.zeros((pages, hkv, 2, D), dtype=torch.bfloat16, device="cuda")}
            st["desc"] = kvshot.make_desc(**attn)
        return st
    if kind == "evict":
        st["k"], st["v"] = _keys((pages, hkv, page, D), g), _randn((pages, hkv, page, D), g)
        kept, counts = _kept(case)
        out_table, out_ids = _table(counts, page, rng)
        st |= {"kept": _int(kept), "counts": _int(counts), "table_out": _int(out_table), "pages_out": len(out_ids),
               "weights": torch.exp(2 * torch.randn((c, max(1, int(lens.max()))), generator=g, device="cuda"))}
        free = ids[int((-(-lens // page)).sum()):]
        st["free"] = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
        st["free"][:len(free)] = _int(free)
        st["free_count"] = _int([len(free)])
        if own:
            zeros = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
            shape = (st["pages_out"], hkv, page, D)
            st["out"] = {"k": zeros(*shape), "v": zeros(*shape), "lens": zeros(c, dtype=torch.int32),
                         "weights": zeros(c, case["keep"], dtype=torch.float32), "free": st["free"].clone(),
                         "free_count": zeros(1, dtype=torch.int32)}
            st["desc"] = kvshot.make_evict_desc(
                num_caches=c, hkv=hkv, page_size=page, max_pages_per_seq=st["table"].shape[1], num_pages=pages,
                max_pages_out=st["table_out"].shape[1], num_pages_out=st["pages_out"], max_kept=case["keep"],
                weights_len=st["weights"].shape[1], weights_len_out=case["keep"], num_free=pages, err_flag=err)
        return st
    hq, nq = case["hq"], case["query"]
    st["q"] = _randn((c, nq, hq, D), g)
    if kind == "scores":
        centre, half = _keys((pages, hkv, D), g).float(), 1.5 * _keys((pages, hkv, D), g).float().abs()
        st["bounds"] = torch.stack([centre - half, centre + half], dim=2).to(torch.bfloat16)
        if own:
            st["out"] = {"scores": torch.zeros((c, nq, hkv, st["table"].shape[1]), device="cuda")}
            st["desc"] = kvshot.make_desc(**attn)
        return st
    if kind == "weights":
        width = max(1, int(lens.max()))
        st["k"] = _keys((pages, hkv, page, D) if page else (c, hkv, st["l_cap"], D), g)
        st["lse"] = _logsumexp(st, 1.0 / math.sqrt(D))
        live = torch.arange(width, device="cuda") < st["lens"][:, None]
        st["weights"] = torch.exp(2 * torch.randn((c, width), generator=g, device="cuda")) * live
        if own:
            st["out"] = {"weights": torch.zeros((c, width), device="cuda")}
            st["desc"] = kvshot.make_desc(**attn)
        return st
    # sparse
    n, seqs = case["nodes"], case["seqs"]
    st["k"], st["v"] = _keys((pages, hkv, page, D), g), _randn((pages, hkv, page, D), g)
    picks, counts = _picks(case)
    st["picks"], st["counts"] = _int(picks), _int(counts)
    st["parent"] = None
    if case["width"]:
        w = case["width"]
        i = np.arange(n)
        st["parent"] = _int(np.where(i < w, -1, (i // w - 1) * w + rng.integers(0, w, size=(seqs, n))))
    slots = -(-n // 8) * 8
    st["draft_k"], st["draft_v"] = _keys((c, hkv, slots, D), g), _randn((c, hkv, slots, D), g)
    if own:
        st["out"] = {"out": torch.empty_like(st["q"]), "lse": torch.empty((c, nq, hq), device="cuda")}
        attn |= dict(n_nodes=n, n_max=slots, tree=case["width"] > 0)
        st["desc"] = kvshot.make_desc(**attn)
        size = kvshot.draft_attn_sparse_workspace_size(st["desc"], case["keep"])
        st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        st["desc"].workspace, st["desc"].workspace_bytes = st["workspace"].data_ptr(), size
    return st


# ------------------------------------------------------------------ one pass

def _plain_bounds(st):
    page, lens = st["case"]["page"], st["lens"]
    out = torch.zeros((*st["k"].shape[:2], 2, D), dtype=torch.bfloat16, device="cuda")
    col = torch.arange(st["table"].shape[1], device="cuda")
    live = (col * page < lens[:, None]) & ((col + 1) * page > st["from"][:, None])   # the pages that hold new tokens
    c, p = torch.nonzero(live, as_tuple=True)
    ids = st["table"][c, p].long()
    valid = (p[:, None] * page + torch.arange(page, device="cuda") < lens[c][:, None])[:, None, :, None]
    for i in range(0, len(ids), 1 << 13):
        j = slice(i, i + (1 << 13))
        k = st["k"][ids[j]].float()
        low = torch.where(valid[j], k, math.inf).amin(2)
        high = torch.where(valid[j], k, -math.inf).amax(2)
        out[ids[j]] = torch.stack([low, high], dim=2).to(torch.bfloat16)
    return {"bounds": out}


def _plain_scores(st):
    case = st["case"]
    c, hq, hkv, nq = case["caches"], case["hq"], case["hkv"], case["query"]
    b = st["bounds"][st["table"].long()].float()                             # [C, pages, hkv, 2, 128]
    low, high = b[:, :, :, 0].permute(0, 2, 3, 1), b[:, :, :, 1].permute(0, 2, 3, 1)
    q = st["q"].float().reshape(c, nq, hkv, hq // hkv, D).permute(0, 2, 1, 3, 4).reshape(c, hkv, -1, D)
    s = torch.matmul(q.clamp(min=0), high) + torch.matmul(q.clamp(max=0), low)
    s = s.reshape(c, hkv, nq, hq // hkv, -1).amax(3).transpose(1, 2) * (1.0 / math.sqrt(D))
    live = torch.arange(s.shape[-1], device="cuda") * case["page"] < st["lens"][:, None]
    return {"scores": torch.where(live[:, None, None], s, torch.zeros_like(s))}


def _plain_select(st):
    case, s = st["case"], st["scores"]
    n = ((st["lens"] + case["unit"] - 1) // case["unit"]).repeat_interleave(case["per"])[:, None].long()
    i = torch.arange(s.shape[1], device="cuda").expand_as(s)
    forced = (i < case["first"]) | (i >= n - case["last"])
    rank = torch.where(i >= n, 2, torch.where(forced, 0, 1))                 # 0: kept whatever its score
    order = torch.sort(torch.where(rank == 1, s, -math.inf), dim=1, descending=True, stable=True).indices
    order = order.gather(1, torch.sort(rank.gather(1, order), dim=1, stable=True).indices)[:, :case["keep"]]
    count = n.clamp(max=case["keep"])
    picked = torch.where(torch.arange(order.shape[1], device="cuda") < count, order, s.shape[1])
    picked = torch.sort(picked, dim=1).values
    picks = torch.full((len(s), case["keep"]), -1, dtype=torch.int32, device="cuda")
    picks[:, :order.shape[1]] = torch.where(picked < s.shape[1], picked, -1).int()
    return {"picks": picks, "counts": count[:, 0].int()}


def _ancestors(parent, n, seqs):
    """[B, N, N]: whether node j is node i or one of its ancestors."""
    i = torch.arange(n, device="cuda")
    up = parent.long() if parent is not None else (i - 1)[None, :].expand(seqs, n)
    step = (up[:, :, None] == i).double() + torch.eye(n, dtype=torch.float64, device="cuda")
    return torch.linalg.matrix_power(step, n) > 0


def _plain_sparse(st):
    case, page = st["case"], st["case"]["page"]
    c, hq, hkv, n, nq = _count(case), case["hq"], case["hkv"], case["nodes"], case["query"]
    g, keep = hq // hkv, case["keep"]
    see = _ancestors(st["parent"], n, case["seqs"]).repeat_interleave(case["layers"], 0)[:, n - nq:]
    out = torch.empty((c, nq, hq, D), device="cuda")
    lse = torch.empty((c, nq, hq), device="cuda")
    head = torch.arange(hkv, device="cuda")[None, :, None]
    offset = torch.arange(page, device="cuda")
    for i in range(c):
        picks = st["picks"][i].long()                                        # [Nq, hkv, keep]
        at = picks.clamp(min=0)
        ids = st["table"][i].long()[at]
        seen = (picks >= 0)[..., None] & (at[..., None] * page + offset < st["lens"][i])
        seen = torch.cat([seen.reshape(nq, hkv, -1), see[i][:, None].expand(nq, hkv, n)], dim=2)
        draft = lambda x: x[i, :, :n].float()[None].expand(nq, hkv, n, D)  # noqa: E731
        pages = lambda x: x[ids, head].float().reshape(nq, hkv, keep * page, D)  # noqa: E731
        k = torch.cat([pages(st["k"]), draft(st["draft_k"])], dim=2)
        v = torch.cat([pages(st["v"]), draft(st["draft_v"])], dim=2)
        q = st["q"][i].float().reshape(nq, hkv, g, D)
        s = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
        s = s.masked_fill(~seen[:, :, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        z = p.sum(-1, keepdim=True)
        out[i] = (torch.matmul(p, v) / z).reshape(nq, hq, D)
        lse[i] = (top + torch.log(z)).reshape(nq, hq)
    return {"out": out.to(torch.bfloat16), "lse": lse}


def _plain_weights(st):
    case = st["case"]
    hq, hkv, nq = case["hq"], case["hkv"], case["query"]
    out = torch.zeros_like(st["weights"])
    for c, n in enumerate(st["host_lens"]):
        q = st["q"][c].float().reshape(nq, hkv, hq // hkv, D).permute(1, 0, 2, 3).reshape(hkv, -1, D)
        z = st["lse"][c].reshape(nq, hkv, hq // hkv).permute(1, 0, 2).reshape(hkv, -1, 1)
        s = torch.matmul(q, _keys_of(st, c).float().transpose(1, 2)) * (1.0 / math.sqrt(D))
        out[c, :n] = case["decay"] * st["weights"][c, :n] + torch.exp(s - z).sum((0, 1))
    return {"weights": out}


def _plain_evict(st):
    case, page = st["case"], st["case"]["page"]
    keep, kept, counts = case["keep"], st["kept"].long(), st["counts"]
    shape = (st["pages_out"], case["hkv"], page, D)
    out = {x: torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for x in ("k", "v")}
    c, i = torch.nonzero(torch.arange(keep, device="cuda") < counts[:, None], as_tuple=True)
    src, at = kept[c, i], (st["table_out"][c, i // page].long(), i % page)
    page_in, off_in = st["table"][c, src // page].long(), src % page
    for x in ("k", "v"):
        out[x][at[0], :, at[1]] = st[x][page_in, :, off_in]
    weights = torch.zeros((len(counts), keep), device="cuda")
    weights[c, i] = st["weights"][c, src]
    # the pages behind those that the kept tokens take, cache after cache
    col = torch.arange(st["table"].shape[1], device="cuda")
    gone = (col * page < st["lens"][:, None]) & (col * page >= counts[:, None])
    rank = torch.cumsum(gone.reshape(-1), 0).reshape(gone.shape) - 1
    free = st["free"].clone()
    free[(st["free_count"] + rank)[gone].long()] = st["table"][gone]
    return {**out, "lens": counts.clone(), "weights": weights, "free": free,
            "free_count": (st["free_count"] + gone.sum()).int()}


def run(state):
    st, case = state, state["case"]
    kind = case["kind"]
    if own:
        from paper_2604_26412_gb300 import kvshot
        o, d = st["out"], st["desc"]
        if kind == "bounds":
            kvshot.page_bounds(d, st["k"], st["table"], st["lens"], st["from"], o["bounds"])
        elif kind == "scores":
            kvshot.page_scores(d, st["q"], st["bounds"], st["table"], st["lens"], o["scores"])
        elif kind == "select":
            kvshot.select_top(d, st["scores"], st["lens"], o["picks"], o["counts"])
        elif kind == "sparse":
            kvshot.draft_attn_sparse(d, st["q"], st["k"], st["v"], st["table"], st["lens"], st["picks"], st["counts"],
                                     case["keep"], st["draft_k"], st["draft_v"], st["parent"], o["out"], o["lse"])
        elif kind == "weights":
            kvshot.key_weights(d, st["q"], st["k"], st["table"], st["lens"], st["lse"], case["decay"],
                               st["weights"].shape[1], st["weights"], o["weights"])
        else:
            kvshot.cache_evict(d, st["k"], st["v"], st["table"], st["lens"], st["kept"], st["counts"], st["weights"],
                               o["k"], o["v"], st["table_out"], o["lens"], o["weights"], o["free"], st["free_count"],
                               o["free_count"])
        return {**o, "err": st["err"]}
    plain = {"bounds": _plain_bounds, "scores": _plain_scores, "select": _plain_select, "sparse": _plain_sparse,
             "weights": _plain_weights, "evict": _plain_evict}[kind]
    return {**plain(st), "err": st["err"]}


def work(case):
    kind, lens = case["kind"], _lens(case)
    c, page = len(lens), case.get("page", 0)
    total, row = int(lens.sum()), 2 * D
    if kind == "bounds":
        start = np.maximum(0, lens - case["new"]) // page * page if case["new"] else np.zeros_like(lens)
        pages = int((-(-lens // page) - start // page).sum())
        return {"bytes": int((lens - start).sum()) * case["hkv"] * row + pages * (case["hkv"] * 2 * row + 4) + 8 * c,
                "flops": 0}
    if kind == "select":
        entries = int((-(-lens // case["unit"])).sum()) * case["per"]
        kept = int(np.minimum(-(-lens // case["unit"]), case["keep"]).sum()) * case["per"]
        return {"bytes": 4 * (entries + kept + c * case["per"] + c), "flops": 0}
    hkv = case["hkv"]
    if kind == "evict":
        kept = int(np.minimum(lens, case["keep"]).sum())
        gone = int((-(-lens // page) - -(-np.minimum(lens, case["keep"]) // page)).sum())
        return {"bytes": kept * (hkv * 4 * row + 12) + 8 * gone + 12 * c, "flops": 0}
    hq, nq = case["hq"], case["query"]
    table = 4 * int((-(-lens // page)).sum()) if page else 0
    if kind == "scores":
        pages = int((-(-lens // page)).sum())
        return {"bytes": pages * hkv * (2 * row + 4 * nq) + c * nq * hq * row + table + 4 * c,
                "flops": 4 * D * hq * nq * pages}
    if kind == "weights":
        return {"bytes": total * (hkv * row + 8) + c * nq * hq * (row + 4) + table + 4 * c,
                "flops": 2 * D * hq * nq * total}
    # sparse: each page that some node of the cache selected is read once for that KV head
    picks, counts = _picks(case)
    n, keys, pairs = case["nodes"], 0, 0
    for i in range(c):
        for h in range(hkv):
            for p in [np.unique(picks[i, :, h])]:
                p = p[p >= 0]
                keys += int(np.minimum(page, lens[i] - p * page).sum())
    pairs = int(counts.sum()) * page + c * nq * hkv * n
    return {"bytes": keys * 2 * row + c * n * hkv * 2 * row + c * nq * hq * (2 * row + 4) + 4 * int(counts.sum())
            + 4 * counts.size + 4 * c + (4 * case["seqs"] * n if case["width"] else 0),
            "flops": 4 * D * (hq // hkv) * pairs}


# ------------------------------------------------------------------ the same in 64 bits

def _exact_select(st):
    case, s = st["case"], st["scores"].double().cpu().numpy()
    picks, counts = np.full((len(s), case["keep"]), -1, np.int32), np.zeros(len(s), np.int32)
    for r in range(len(s)):
        n = -(-int(st["host_lens"][r // case["per"]]) // case["unit"])
        m = min(n, case["keep"])
        must = set(range(min(case["first"], n))) | set(range(max(0, n - case["last"]), n))
        for i in np.argsort(-s[r, :n], kind="stable"):
            if len(must) >= m:
                break
            must.add(int(i))
        picks[r, :m] = sorted(must)
        counts[r] = m
    return {"picks": picks, "counts": counts, "err": None}


def _exact_evict(st):
    case, page = st["case"], st["case"]["page"]
    kept, counts = st["kept"].cpu().numpy(), st["counts"].cpu().numpy()
    table, table_out, lens = st["table"].cpu().numpy(), st["table_out"].cpu().numpy(), st["host_lens"]
    out = {x: torch.zeros((st["pages_out"], case["hkv"], page, D), dtype=torch.float64, device="cuda") for x in ("k", "v")}
    weights = torch.zeros((len(counts), case["keep"]), dtype=torch.float64, device="cuda")
    free = st["free"].cpu().numpy().copy()
    f = int(st["free_count"][0])
    for c, m in enumerate(counts):
        rows = torch.from_numpy(kept[c, :m].astype(np.int64)).cuda()
        used = max(1, -(-int(lens[c]) // page))
        ids = torch.from_numpy(table[c, :used].astype(np.int64)).cuda()
        for x in ("k", "v"):
            whole = st[x][ids].double().transpose(0, 1).reshape(case["hkv"], -1, D)[:, rows]
            for p in range(0, int(m), page):
                part = whole[:, p:p + page]
                out[x][table_out[c, p // page], :, :part.shape[1]] = part
        weights[c, :m] = st["weights"][c, rows].double()
        for p in range(-(-int(m) // page), -(-int(lens[c]) // page)):
            free[f] = table[c, p]
            f += 1
    return {**out, "lens": counts, "weights": weights, "free": free, "free_count": np.array([f], np.int32), "err": None}


def exact(case, seed):
    st = prepare(case, seed)
    kind, lens, page = case["kind"], st["host_lens"], case.get("page", 0)
    if kind == "select":
        return _exact_select(st)
    if kind == "evict":
        return _exact_evict(st)
    hkv = case["hkv"]
    table = st["table"].cpu().numpy() if page else None
    if kind == "bounds":
        out = torch.zeros((*st["k"].shape[:2], 2, D), dtype=torch.float64, device="cuda")
        start = st["from"].cpu().numpy()
        for c, n in enumerate(lens):
            for p in range(int(start[c]) // page, -(-int(n) // page)):
                rows = st["k"][table[c, p], :, :min(page, int(n) - p * page)].double()
                out[table[c, p], :, 0], out[table[c, p], :, 1] = rows.min(1).values, rows.max(1).values
        return {"bounds": out, "err": None}
    hq, nq, scale = case["hq"], case["query"], 1.0 / math.sqrt(D)
    g = hq // hkv
    if kind == "scores":
        out = torch.zeros((len(lens), nq, hkv, st["table"].shape[1]), dtype=torch.float64, device="cuda")
        for c, n in enumerate(lens):
            used = -(-int(n) // page)
            b = st["bounds"][st["table"][c, :used].long()].double()          # [pages, hkv, 2, 128]
            for r in range(nq):
                for h in range(hkv):
                    q = st["q"][c, r, h * g:(h + 1) * g].double()[:, None]
                    s = torch.maximum(q * b[None, :, h, 0], q * b[None, :, h, 1]).sum(-1)
                    out[c, r, h, :used] = s.max(0).values * scale
        return {"scores": out, "err": None}
    if kind == "weights":
        out = torch.zeros(st["weights"].shape, dtype=torch.float64, device="cuda")
        for c, n in enumerate(lens):
            k = _keys_of(st, c).double()
            w = case["decay"] * st["weights"][c, :n].double()
            for h in range(hq):
                s = st["q"][c, :, h].double() @ k[h // g].T * scale - st["lse"][c, :, h].double()[:, None]
                w = w + torch.exp(s).sum(0)
            out[c, :n] = w
        return {"weights": out, "err": None}
    n = case["nodes"]
    out = torch.empty((len(lens), nq, hq, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((len(lens), nq, hq), dtype=torch.float64, device="cuda")
    parent = st["parent"].cpu().numpy() if st["parent"] is not None else None
    if len(lens) * nq * hkv > 4096:
        return None
    picks, counts = st["picks"].cpu().numpy(), st["counts"].cpu().numpy()
    for c, length in enumerate(lens):
        line = []  # of each node: the nodes from it to its root
        for i in range(n):
            up = int(parent[c // case["layers"], i]) if parent is not None else i - 1
            line.append([i] + (line[up] if up >= 0 else []))
        used = max(1, -(-int(length) // page))
        k_all, v_all = (_gather(st[x], st["table"][c:c + 1, :used], page)[0] for x in ("k", "v"))
        for r in range(nq):
            own_line = torch.tensor(line[n - nq + r], device="cuda")
            for h in range(hkv):
                at = (picks[c, r, h, :counts[c, r, h], None].astype(np.int64) * page + np.arange(page)).reshape(-1)
                at = torch.from_numpy(at[at < length]).cuda()
                k = torch.cat([k_all[h, at], st["draft_k"][c, h, own_line]]).double()
                v = torch.cat([v_all[h, at], st["draft_v"][c, h, own_line]]).double()
                s = st["q"][c, r, h * g:(h + 1) * g].double() @ k.T * scale
                z = torch.logsumexp(s, dim=1)
                out[c, r, h * g:(h + 1) * g] = torch.exp(s - z[:, None]) @ v
                lse[c, r, h * g:(h + 1) * g] = z
    return {"out": out, "lse": lse, "err": None}
