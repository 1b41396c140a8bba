"""Sparse attention: draft nodes that no query row sees may hold anything and count as nothing.

Trees of which some branches have no node among the query rows, those branches' K and V spoilt, through the kernel of shared
pages and the one with a CTA for each node.  Results and bounds as in tests/test_gpu_partial.py.
"""
import numpy as np
import pytest
import torch

from oracle import partial
from paper_2604_26412_gb300 import kvshot

from .partial_problems import Problem, f64
from .test_gpu_partial import SHARED, run_sparse

pytestmark = pytest.mark.gpu

CASES = {
    "shared": dict(SHARED["tree"]),
    "shared, one head": dict(SHARED["one head"], query=40),
    "shared, blocks of 3 nodes": dict(lens=list(range(0, 530, 10)), page=64, hq=34, hkv=2, nodes=30, query=5, tree=True),
    "a CTA for each node": dict(lens=[3, 333, 90], page=16, nodes=12, query=2, tree=True),
}


def unseen(p):
    """Draft slots of every cache that are no query node's own and no ancestor's."""
    out = []
    for c in range(len(p.lens)):
        seen = set()
        for n in range(p.N - p.Nq, p.N):
            seen.update(partial.line_of(p.parent[c // p.layers], n))
        out.append(sorted(set(range(p.N)) - seen))
    return out


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
def test_branches_that_no_row_sees(name, what):
    p = Problem(**CASES[name], seed=17)
    picks, counts = p.random_picks(16, seed=17)
    want = run_sparse(p, picks, counts)
    hidden = unseen(p)
    assert sum(map(len, hidden)) > 0
    for c, slots in enumerate(hidden):
        p.dk[c, :, slots] = p.dv[c, :, slots] = what
    got = run_sparse(p, picks, counts)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("name", CASES)
def test_one_branch_of_a_level_does_not_reach_another(name):
    """NaN in the V of one node that one query row alone sees: the other KV heads' rows, and the other caches', stay as they
    are; of that head, rows may have it."""
    p = Problem(**CASES[name], seed=18)
    picks, counts = p.random_picks(16, seed=18)
    want = run_sparse(p, picks, counts)
    c, g = len(p.lens) - 1, p.hq // p.hkv
    p.dv[c, 0, p.N - 1] = float("nan")
    ws = p.workspace(16)
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    kvshot.draft_attn_sparse(p.desc, p.q, p.k, p.v, p.t_table, p.t_lens, p.ints(picks), p.ints(counts), 16, p.dk, p.dv,
                             p.t_parent, out, lse)
    torch.cuda.synchronize()
    del ws
    keep = torch.ones(out.shape[:3], dtype=torch.bool, device="cuda")
    keep[c, :, :g] = False
    assert torch.equal(out[keep], want[0][keep]) and torch.equal(lse, want[1])
    assert bool(torch.isnan(out[c, -1, :g]).all())
    assert np.isfinite(lse.cpu().numpy()).all()


@pytest.mark.parametrize("name", CASES)
def test_keys_of_minus_infinity_weigh_nothing(name):
    """Scores of -inf, of the nodes' own keys and of some of a page's, beside finite ones.  Bounds as in tests/test_gpu_partial.py, of
    the finite keys: a weight of 0 is exact."""
    p = Problem(**CASES[name], seed=19)
    picks, counts = p.random_picks(16, seed=19)
    p.q[..., 0] = p.q[..., 0].abs() + 1
    own, k0 = slice(p.N - p.Nq, p.N), [int(x) for x in p.table[:, 0] if x >= 0]
    p.dk[:, :, own, 0] = 0
    p.k[k0, :, ::3, 0] = 0
    mag = oracle(p, picks, counts)[3]
    p.dk[:, :, own, 0] = float("-inf")
    p.k[k0, :, ::3, 0] = float("-inf")
    with np.errstate(invalid="ignore"):  # (rows of -inf alone have no softmax)
        want, z, spread, _ = oracle(p, picks, counts)
    ws = p.workspace(16)
    out, lse = torch.empty_like(p.q), torch.empty(p.q.shape[:3], device="cuda")
    kvshot.draft_attn_sparse(p.desc, p.q, p.k, p.v, p.t_table, p.t_lens, p.ints(picks), p.ints(counts), 16, p.dk, p.dv,
                             p.t_parent, out, lse)
    torch.cuda.synchronize()
    assert int(p.err.item()) == 0
    del ws
    seen = np.isfinite(z)
    assert seen.sum() > seen.size // 2
    tol = 2.0 ** -16 * mag + 2.0 ** -18
    assert np.all(np.abs(f64(lse) - z)[seen] <= tol[seen])
    assert np.all((np.abs(f64(out) - want) <= (2.0 ** -7 + 2 * tol[..., None]) * spread)[seen])


def oracle(p, picks, counts):
    return partial.attn_sparse(f64(p.q), f64(p.k), f64(p.v), p.table, p.lens, picks, counts, f64(p.dk), f64(p.dv), p.parent,
                               p.layers, p.N, p.scale)
