"""Drafting over selected pages of a cache that evictions change: the bounds of every selection follow the moved keys, eagerly
and in a captured graph."""
import gc

import numpy as np
import pytest
import torch

from oracle import partial
from paper_2604_26412_gb300.partial import PageSelection, TokenWeights
from paper_2604_26412_gb300.step import DraftStep

from .partial_problems import f64
from .test_gpu_partial_step import check_levels, inputs, picked

pytestmark = pytest.mark.gpu

LENS = (200, 0, 130, 1000)


def check_bounds(inp, pages):
    """The pages of the present lengths, exactly."""
    torch.cuda.synchronize()
    lens, table = inp.seq_lens.cpu().numpy(), inp.page_table.cpu().numpy()
    want = partial.page_bounds(f64(inp.target_k), table, lens, 0 * lens, f64(pages.bounds))
    assert np.array_equal(f64(pages.bounds), want)
    assert pages.error_code() == 0


@pytest.mark.parametrize("side_stream", [False, True])
def test_bounds_follow_an_eviction(side_stream):
    inp = inputs(lens=LENS)
    pages, more, w = PageSelection(inp, keep=5), PageSelection(inp, keep=3, first=0, last=1), TokenWeights(inp)
    steps = [DraftStep(inp, pages=x) for x in (pages, more)]
    DraftStep(inp, weights=w).run()
    before = pages.bounds.clone()
    stream = torch.cuda.Stream() if side_stream else None
    torch.cuda.synchronize()
    w.evict(100, first=4, last=20, stream=stream)
    check_bounds(inp, pages)
    check_bounds(inp, more)
    assert not torch.equal(pages.bounds, before)
    for step in steps:
        step.run()
        torch.cuda.synchronize()
        check_levels(step, lambda i: picked(step, i))
        lens, table = inp.seq_lens.cpu().numpy(), inp.page_table.cpu().numpy()
        bounds = partial.page_bounds(f64(inp.target_k), table, lens, 0 * lens, 0 * f64(pages.bounds))
        width = table.shape[1]
        live = (np.arange(width) * 16 < lens[:, None])[:, None, None]
        for i, got in enumerate(step.scores):
            want, mag = partial.page_scores(f64(step.q_rot[i]), bounds, table, lens, 16, 128 ** -0.5, np.zeros(got.shape))
            assert np.all((np.abs(f64(got) - want) <= 2.0 ** -14 * mag) | ~live)


def test_growth_after_an_eviction():
    """Tokens behind the kept ones: update() from the lengths of the evicted cache, as after any growth."""
    inp = inputs(lens=LENS)
    pages, w = PageSelection(inp, keep=5), TokenWeights(inp)
    w.evict(70, first=4, last=20)
    before = inp.seq_lens.clone()
    inp.seq_lens += torch.tensor([5, 0, 60, 100], dtype=torch.int32, device="cuda")  # (in pages that the tables still name)
    for c, n in enumerate(inp.seq_lens.tolist()):
        for j in range(int(before[c]), n):
            inp.target_k[inp.page_table[c, j // 16].long(), :, j % 16] = c + j / 64
    pages.update(before)
    check_bounds(inp, pages)


def test_a_captured_eviction_keeps_the_bounds():
    inp = inputs(lens=LENS)
    pages, w = PageSelection(inp, keep=5), TokenWeights(inp)
    step = DraftStep(inp, pages=pages)
    state = (inp.target_k, inp.target_v, inp.seq_lens, pages.bounds, w.weights, w.free_pages, w.free_count)
    w.weights.copy_(torch.rand(w.weights.shape, device="cuda"))
    start = [x.clone() for x in state]

    def work():
        w.evict(90, 2, 16)
        step.run()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        work()
    stream.synchronize()
    want = [x.clone() for x in (*state, *step.out, *step.lse)]

    def reset():
        for x, y in zip(state, start):
            x.copy_(y)
        torch.cuda.synchronize()
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        work()
    reset()
    graph.replay()
    torch.cuda.synchronize()
    for x, y in zip((*state, *step.out, *step.lse), want):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    check_bounds(inp, pages)


def test_a_captured_eviction_keeps_its_selections_alive():
    """A graph writes bounds whose selection its user has let go of: that memory is not another tensor's meanwhile."""
    inp = inputs(lens=LENS)
    pages, w = PageSelection(inp, keep=5), TokenWeights(inp)
    w.evict(190, 2, 16)  # (so that the capture allocates nothing)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w.evict(190, 2, 16)
    at, size = pages.bounds.data_ptr(), pages.bounds.shape
    del pages
    gc.collect()
    others = [torch.full(size, 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(8)]
    assert at not in [x.data_ptr() for x in others]
    graph.replay()
    torch.cuda.synchronize()
    assert all(bool((x == 7).all()) for x in others)


def test_a_selection_that_is_gone_costs_nothing():
    inp = inputs(lens=LENS)
    w = TokenWeights(inp)
    pages = PageSelection(inp, keep=5)
    del pages
    gc.collect()
    assert len(inp.selections) == 0
    w.evict(100)
    assert w.error_code() == 0
