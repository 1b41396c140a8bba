"""4-bit cache attention: what no query row sees may hold anything and counts as nothing.

The cases of tests/test_gpu_kv4.py with, afterwards, NaN in every draft slot that no query row sees, NaN scales in every
such token of the prefix, and an invalid id in the table for every page whose tokens are all hidden (of a tree: hidden
from a node of depth 1).  Results and bounds as there: nothing of it may show.
"""
import numpy as np
import pytest
import torch

from oracle import kv4
from paper_2604_26412_gb300 import kvshot
from tests.test_gpu_kv4 import D, LSE_MAX_ABS, OUT_MAX_ABS, OUT_REL_L2, Case, _i32, _tree

pytestmark = pytest.mark.gpu

# hq, hkv, nodes, query: 8, 16, 32, 48, 64 and 4 x 40 query rows per KV head
ROWS = [(8, 2, 12, 2), (8, 2, 16, 4), (8, 2, 20, 8), (8, 2, 24, 12), (8, 2, 32, 16), (8, 2, 60, 40)]


def _poison(case, drafts=True, prefix=True, pages=True):
    """Returns how many draft slots, prefix tokens and pages it has spoilt."""
    kc, ks, vc, vs = kv4.unpack(case.cache.cpu().numpy())
    dk, dv = case.dk.cpu(), case.dv.cpu()
    table = case.table.cpu().numpy() if case.table is not None else None
    spoilt = [0, 0, 0]
    for c, length in enumerate(case.lens):
        par = case.parent[c // (len(case.lens) // case.seqs)] if case.parent is not None else None
        lines = kv4.node_lines(par, case.n)
        seen, nodes = set(), set()
        for i in range(case.n - case.nq, case.n):
            js, ms = kv4.visible(length, lines, i, case.window, case.sinks)
            seen.update(js)
            nodes.update(ms)
        for m in set(range(case.n)) - nodes if drafts else ():
            dk[c, :, m] = dv[c, :, m] = float("nan")
            spoilt[0] += 1
        for j in set(range(length)) - seen if prefix else ():
            at = (table[c, j // case.page] if table is not None else c, slice(None), j % case.page)
            ks[at] = vs[at] = 0x7F
            spoilt[1] += 1
        if table is None or not pages:
            continue
        least = 1 if par is not None else case.n - case.nq + 1
        first = length + least - case.window if case.window else 0
        for pg in range(-(-length // case.page)):
            if pg * case.page >= case.sinks and min(length, (pg + 1) * case.page) <= first:
                table[c, pg] = -9
                spoilt[2] += 1
    case.cache = torch.from_numpy(kv4.pack(kc, ks, vc, vs)).cuda()
    case.dk, case.dv = dk.cuda(), dv.cuda()
    if table is not None:
        case.table = _i32(table)
    return spoilt


@pytest.mark.parametrize("hq,hkv,nodes,query", ROWS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (3, 0)])
def test_draft_nodes_that_no_row_sees(hq, hkv, nodes, query, window, sinks):
    """Branches that the query nodes do not descend from, and (with a window) ancestors that lie too far back."""
    rng = np.random.default_rng(nodes)
    case = Case([150, 0, 40], hq=hq, hkv=hkv, nodes=nodes, query=query, parent=_tree(rng, 3, nodes, 4), window=window,
                sinks=sinks, seed=nodes)
    assert _poison(case, prefix=False, pages=False)[0] > 0
    case.check()


@pytest.mark.parametrize("hq,hkv,nodes,query", ROWS)
def test_draft_nodes_of_a_chain_beyond_the_window(hq, hkv, nodes, query):
    case = Case([150, 0, 40], hq=hq, hkv=hkv, nodes=nodes + 30, query=query, window=6, seed=nodes)
    assert _poison(case, prefix=False, pages=False)[0] > 0
    case.check()


@pytest.mark.parametrize("hq,hkv,nodes,query", ROWS)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("window,sinks,page", [(40, 0, 16), (40, 3, 0), (130, 20, 32), (100, 130, 256)])
def test_prefix_tokens_that_no_row_sees(hq, hkv, nodes, query, tree, window, sinks, page):
    """NaN scales up to the first token that the shallowest query row sees, which of a tree's deep level is not a child of
    the last verified token."""
    rng = np.random.default_rng(nodes)
    par = _tree(rng, 2, nodes, 2) if tree else None
    case = Case([451, 700], hq=hq, hkv=hkv, nodes=nodes, query=query, parent=par, window=window, sinks=sinks, page=page,
                seed=nodes + page)
    assert _poison(case, drafts=False, pages=False)[1] > 0
    case.check()


@pytest.mark.parametrize("hq,hkv,nodes,query", ROWS)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("window,sinks,page", [(40, 0, 16), (40, 3, 16), (130, 20, 32), (200, 130, 48), (77, 0, 64),
                                               (100, 1, 128), (60, 0, 256), (5, 2, 16)])
def test_pages_that_no_row_sees_are_not_looked_up(hq, hkv, nodes, query, tree, window, sinks, page):
    rng = np.random.default_rng(nodes)
    par = _tree(rng, 3, nodes, 3) if tree else None
    case = Case([451, 1000, 64], hq=hq, hkv=hkv, nodes=nodes, query=query, parent=par, window=window, sinks=sinks,
                page=page, seed=nodes + page)
    assert _poison(case)[2] > 0
    case.check()


def test_a_window_shorter_than_the_chain_sees_no_prefix():
    for rows in ROWS:
        hq, hkv, _, query = rows
        for sinks in (0, 3):
            case = Case([128, 130, 451], hq=hq, hkv=hkv, nodes=query + 20, query=query, window=9, sinks=sinks, seed=query)
            assert min(_poison(case)) > 0
            case.check()


# ------------------------------------------------------------------ very long contexts

@pytest.mark.parametrize("group,length", [(8, 3 * 2 ** 27 + 77), (16, 3 * 2 ** 26 + 77), (32, 3 * 2 ** 25 + 77),
                                          (64, 3 * 2 ** 24 + 77), (200, 3 * 2 ** 22 + 77)])
@pytest.mark.parametrize("sinks", [5, 130])
def test_a_window_at_the_end_of_a_very_long_context(group, length, sinks):
    """Hidden keys in the sinks' last tile, so far from the window that (distance x rows of a node) passes 2^31.  One page
    of 2^20 tokens stands for all of them; against the same attention to the sinks and the window's tokens alone."""
    page, window, nodes = 1 << 20, 100, 3
    gen = torch.Generator("cuda").manual_seed(group)
    cache = torch.randint(0, 256, (page // 16, 2304), dtype=torch.uint8, device="cuda", generator=gen)
    cache[:, 2048:] = torch.randint(0x30, 0x40, (page // 16, 256), dtype=torch.uint8, device="cuda", generator=gen)
    table = torch.zeros((1, -(-length // page)), dtype=torch.int32, device="cuda")
    bf = lambda *s: torch.randn(s, device="cuda", generator=gen).to(torch.bfloat16)  # noqa: E731
    q, dk, dv = bf(1, nodes, group, D), bf(1, 1, nodes, D), bf(1, 1, nodes, D)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = kvshot.make_desc(num_caches=1, num_seqs=1, hq=group, hkv=1, n_nodes=nodes, n_query=1, n_max=nodes,
                            max_seq_len=length, page_size=page, max_pages_per_seq=table.shape[1], num_pages=1, err_flag=err)
    ws = torch.empty(kvshot.draft_attn_kv4_workspace_size(desc, window, sinks), dtype=torch.uint8, device="cuda")
    desc.workspace, desc.workspace_bytes = ws.data_ptr(), ws.numel()
    q = q[:, -1:].contiguous()
    out, lse = torch.empty_like(q), torch.empty((1, 1, group), device="cuda")
    kvshot.draft_attn_kv4(desc, q, cache, table, _i32([length]), dk, dv, None, window, sinks, out, lse)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    near = 160  # tokens before the end, more than the window reaches
    at = np.concatenate([np.arange(sinks), np.arange(length - near, length)]) % page
    parts = kv4.unpack(cache[torch.from_numpy(at // 16).cuda()].cpu().numpy()[None, :, None].swapaxes(0, 1))
    kc, ks, vc, vs = (x[np.arange(len(at)), 0, at % 16] for x in parts)
    k, v = kv4.values(kc, ks, 0)[None], kv4.values(vc, vs, 0)[None]
    ref, ref_lse = kv4.attn(q[0].double().cpu().numpy(), k, v, dk[0].double().cpu().numpy(), dv[0].double().cpu().numpy(),
                            None, window, sinks, D ** -0.5)
    o = out[0].double().cpu().numpy()
    assert np.abs(o - ref).max() <= OUT_MAX_ABS * max(1.0, np.abs(v).max() / 4)
    assert np.linalg.norm(o - ref) <= OUT_REL_L2 * np.linalg.norm(ref)
    assert np.abs(lse[0].double().cpu().numpy() - ref_lse).max() <= LSE_MAX_ABS
