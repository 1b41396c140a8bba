"""4-bit cache attention: what no query row sees may hold anything and counts as nothing.

The cases of tests/test_gpu_kv4.py with, afterwards, NaN in every draft slot that no query row sees, NaN scales in every
such token of the prefix, and an invalid id in the table for every page whose tokens are all hidden (of a tree: hidden
from a node of depth 1).  Results and bounds as there: nothing of it may show.
"""
import numpy as np
import pytest
import torch

from oracle import kv4
from tests.test_gpu_kv4 import Case, _i32, _tree

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
