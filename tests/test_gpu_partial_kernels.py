"""The sizes at which the entry points of drafting over a part of a long cache change their kernels, with the kernel that a call
launches looked up in a captured graph of it: the cases below stay on the paths that they are for.

Results and bounds as in tests/test_gpu_partial.py.
"""
import re
import warnings

import pytest
import torch

from paper_2604_26412_gb300 import kvshot

from .partial_problems import D, Problem
from .test_gpu_partial import run_scores, run_sparse, run_weights

pytestmark = pytest.mark.gpu


@pytest.fixture
def kernels(tmp_path, monkeypatch):
    """kernels(name, f): what f() launches of the library's kernels, where f calls the entry point kvshot.<name> once."""
    def look(name, f):
        launched, call = [], getattr(kvshot, name)

        def captured(*args):
            graph = torch.cuda.CUDAGraph(keep_graph=True)
            with torch.cuda.graph(graph):
                call(*args)
            path = str(tmp_path / "graph.dot")
            with warnings.catch_warnings():  # (it warns that it was called)
                warnings.simplefilter("ignore")
                graph.debug_dump(path)
            launched.extend(sorted(set(re.findall(r"([a-z_]+_kernel)(?=[^a-z_])", open(path).read()))))
            return call(*args)
        monkeypatch.setattr(kvshot, name, captured)
        f()
        monkeypatch.undo()
        return launched
    return look


def bounds_of(p):
    return torch.randn((p.num_pages, p.hkv, 2, D), device="cuda").sort(dim=2).values.to(torch.bfloat16)


# ------------------------------------------------------------ sparse attention

SPARSE = [  # G heads that do not divide 64; 32 rows, 128 picked tokens, two thirds of the SMs: the edges of the rule
    (dict(lens=list(range(0, 530, 10)), page=128, hq=34, hkv=2, nodes=3, query=3), 16, "sparse_shared_kernel"),
    (dict(lens=list(range(0, 530, 10)), page=16, hq=34, hkv=2, nodes=30, query=7, tree=True), 16, "sparse_shared_kernel"),
    (dict(lens=list(range(0, 520, 10)), page=32, hq=58, hkv=2, nodes=4, query=2), 16, "sparse_shared_kernel"),
    (dict(lens=[300] * 13, page=16, nodes=8, query=8), 8, "sparse_shared_kernel"),
    (dict(lens=[300] * 13, page=16, nodes=8, query=8), 7, "sparse_kernel"),
    (dict(lens=[300] * 13, page=16, nodes=7, query=7), 8, "sparse_kernel"),
    (dict(lens=[300] * 12, page=16, nodes=8, query=8), 8, "sparse_kernel"),
]


@pytest.mark.parametrize("case,keep,kernel", SPARSE)
def test_sparse(kernels, case, keep, kernel):
    p = Problem(**case, seed=keep)
    assert kernels("draft_attn_sparse", lambda: run_sparse(p, *p.random_picks(keep, seed=keep))) == [kernel]


# ------------------------------------------------------------ scores

@pytest.mark.parametrize("case,kernel", [
    (dict(lens=[2040] * 20, page=8, hq=34, hkv=2, nodes=5, query=5), "scores_tc_kernel"),
    (dict(lens=[1025] * 64, page=8, nodes=12, query=12), "scores_tc_kernel"),
    (dict(lens=[1025] * 64, page=8, nodes=11, query=11), "scores_kernel"),
    (dict(lens=[1016] * 80, page=8, nodes=12, query=12), "scores_kernel"),
])
def test_scores(kernels, case, kernel):
    p = Problem(**case, seed=3)
    assert kernels("page_scores", lambda: run_scores(p, bounds_of(p))) == [kernel]


# ------------------------------------------------------------ weights

@pytest.mark.parametrize("page", [8, 16, 64, 128, 192, 256])
@pytest.mark.parametrize("query,kernel", [(17, "weights_tc_kernel"), (16, "weights_kernel"), (2, "weights_kernel")])
def test_weights_pages(kernels, page, query, kernel):
    p = Problem([0, 1, 7, 8, 9, 63, 64, 65, 130, 257, 300], page, nodes=query, query=query, seed=page)
    assert kernels("key_weights", lambda: run_weights(p)) == [kernel]


@pytest.mark.parametrize("longest,grouped", [(781, True), (773, True), (765, True), (780, False), (5, True), (1, False)])
@pytest.mark.parametrize("query", [17, 64, 70])
def test_weights_of_a_contiguous_cache(kernels, longest, grouped, query):
    """Rows of l_cap = longest + 3: a multiple of 64, of 8 alone (boxes that end in the next head's rows, or behind the cache),
    and of neither."""
    p = Problem([longest, min(longest, 5), 0, min(longest, 128)], 16, nodes=query, query=query, contiguous=True, seed=query)
    assert (p.desc.l_cap % 8 == 0) == grouped
    assert kernels("key_weights", lambda: run_weights(p, 0.5)) == ["weights_tc_kernel"]


def test_weights_of_many_contiguous_caches(kernels):
    p = Problem([133, 0, 1, 128, 127] * 30, 16, hq=8, hkv=2, nodes=5, query=5, contiguous=True, seed=5)
    assert p.desc.l_cap % 8 == 0
    assert kernels("key_weights", lambda: run_weights(p, 0.5)) == ["weights_tc_kernel"]
