"""Drafting steps over selected pages, with token weights and with eviction between them: append, scores, selection and
attention of every level, eagerly, from a captured graph and on another stream.

Bounds as in tests/test_gpu_partial.py; the appended q and draft K/V are those that the library stored (their own tests
compare them bit for bit).
"""
import numpy as np
import pytest
import torch

from oracle import partial
from paper_2604_26412_gb300 import kvshot
from paper_2604_26412_gb300 import workloads as wl
from paper_2604_26412_gb300.partial import PageSelection, TokenWeights
from paper_2604_26412_gb300.step import DraftStep
from tests.partial_problems import f64

pytestmark = pytest.mark.gpu

SCALE = 128 ** -0.5


def inputs(levels=(2, 3), tree=True, layers=1, lens=(40, 0, 130, 1000), hq=8, hkv=2, seed=3):
    spec = wl.Spec("partial-step", len(lens) // layers, layers, list(lens), list(levels), tree, True, page_size=16, hq=hq,
                   hkv=hkv, seed=seed)
    return wl.make_inputs(spec, "cuda", seed=seed, tail_fill="nan")


def check_levels(step, picks_of):
    """Every level of a step against the 64-bit attention over the pages that picks_of(level) gives."""
    inp, s = step.inp, step.inp.spec
    lens, n0 = inp.seq_lens.cpu().numpy(), 0
    for i, n in enumerate(step.levels):
        n0 += n
        picks, counts = picks_of(i)
        want, z, spread, mag = partial.attn_sparse(
            f64(step.q_rot[i]), f64(inp.target_k), f64(inp.target_v), inp.page_table.cpu().numpy(), lens, picks, counts,
            f64(step.draft_k), f64(step.draft_v), step.parents[i].cpu().numpy() if s.tree else None, s.layers, n0, SCALE)
        tol = 2.0 ** -16 * mag + 2.0 ** -18
        assert np.all(np.abs(f64(step.lse[i]) - z) <= tol), i
        assert np.all(np.abs(f64(step.out[i]) - want) <= (2.0 ** -7 + 2 * tol[..., None]) * spread), i
    assert step.error_code() == 0


def picked(step, i):
    return step.picks[i].cpu().numpy(), step.counts[i].cpu().numpy()


@pytest.mark.parametrize("mode", ["per_depth", "whole"])
@pytest.mark.parametrize("tree,layers", [(True, 1), (True, 2), (False, 1)])
def test_steps_over_selected_pages(mode, tree, layers):
    inp = inputs((2, 3) if tree else (1, 1, 1), tree, layers)
    pages = PageSelection(inp, keep=6, first=1, last=2)
    step = DraftStep(inp, mode=mode, pages=pages)
    step.run()
    torch.cuda.synchronize()
    check_levels(step, lambda i: picked(step, i))
    lens, width = inp.seq_lens.cpu().numpy(), inp.page_table.shape[1]
    for i in range(len(step.levels)):
        # the picks are the best pages by the scores, and the scores bound what they stand for
        rows = step.scores[i].reshape(-1, width).cpu().numpy().astype(np.float64)
        want = partial.select_top(rows, lens, step.levels[i] * 2, 16, 6, 1, 2)
        assert np.array_equal(step.picks[i].reshape(-1, 6).cpu().numpy(), want[0])
        bounds = partial.page_bounds(f64(inp.target_k), inp.page_table.cpu().numpy(), lens, 0 * lens, 0 * f64(pages.bounds))
        score, mag = partial.page_scores(f64(step.q_rot[i]), bounds, inp.page_table.cpu().numpy(), lens, 16, SCALE,
                                         np.zeros(step.scores[i].shape))
        live = (np.arange(width) * 16 < lens[:, None])[:, None, None]
        assert np.all((np.abs(f64(step.scores[i]) - score) <= 2.0 ** -14 * mag) | ~live)
    assert int(pages.err.item()) == 0


def test_a_selection_of_all_pages_is_the_draft_attention():
    inp = inputs()
    step, sparse = DraftStep(inp), DraftStep(inp, pages=PageSelection(inp, keep=63, first=0, last=0))
    step.run()
    sparse.run()
    torch.cuda.synchronize()
    for i in range(len(step.levels)):
        assert (step.out[i].float() - sparse.out[i].float()).abs().max() <= 0.03
        assert (step.lse[i] - sparse.lse[i]).abs().max() <= 1e-3


def test_bounds_follow_a_cache_that_grows():
    inp = inputs(lens=(40, 16, 130, 1000))
    pages = PageSelection(inp, keep=5)
    before = torch.tensor([30, 0, 129, 1000], dtype=torch.int32, device="cuda")
    for c in range(4):  # keys that came after `before`
        for j in range(int(before[c]), inp.spec.seq_lens[c]):
            inp.target_k[inp.page_table[c, j // 16].long(), :, j % 16] += 1
    pages.update(before)
    torch.cuda.synchronize()
    lens = inp.seq_lens.cpu().numpy()
    want = partial.page_bounds(f64(inp.target_k), inp.page_table.cpu().numpy(), lens, 0 * lens, f64(pages.bounds))
    assert np.array_equal(f64(pages.bounds), want)
    with pytest.raises(ValueError):
        pages.update(before.long())
    with pytest.raises(ValueError):
        pages.update(before[:3])


def levels_weights(step, weights, decay):
    inp = step.inp
    for i in range(len(step.levels)):
        weights, _ = partial.key_weights(f64(step.q_rot[i]), f64(inp.target_k), inp.page_table.cpu().numpy(),
                                         inp.seq_lens.cpu().numpy(), f64(step.lse[i]), decay, weights, weights, SCALE)
    return weights


@pytest.mark.parametrize("levels,hq,hkv", [((2, 3), 8, 2), ((12, 12), 8, 2), ((40,), 8, 1)])
def test_weights_and_eviction_between_steps(levels, hq, hkv):
    inp = inputs(levels, lens=(40, 0, 130, 700), hq=hq, hkv=hkv)
    w = TokenWeights(inp, decay=0.5)
    step = DraftStep(inp, weights=w)
    step.run()
    torch.cuda.synchronize()
    want = levels_weights(step, np.zeros(w.weights.shape), 0.5)
    assert np.abs(f64(w.weights) - want).max() <= 1e-4 * want.max()
    # the tokens to keep follow from the weights as the library added them up
    lens, table = inp.seq_lens.cpu().numpy(), inp.page_table.cpu().numpy()
    kept, counts = partial.select_top(f64(w.weights), lens, 1, 1, 100, 4, 20)
    bits = lambda x: x.view(torch.int16).cpu().numpy()  # noqa: E731
    k, v, lens_out, weights, free, count = partial.cache_evict(
        bits(inp.target_k), bits(inp.target_v), table, lens, kept, counts, f64(w.weights), bits(inp.target_k),
        bits(inp.target_v), table, f64(w.weights), w.free_pages.cpu().numpy(), 0)
    w.evict(100, first=4, last=20)
    torch.cuda.synchronize()
    assert np.array_equal(bits(inp.target_k), k) and np.array_equal(bits(inp.target_v), v)
    assert inp.seq_lens.tolist() == lens_out.tolist() == [40, 0, 100, 100]
    assert np.array_equal(f64(w.weights), weights)
    assert np.array_equal(w.free_pages.cpu().numpy(), free) and int(w.free_count.item()) == count == (9 - 7) + (44 - 7)
    step.run()
    torch.cuda.synchronize()

    def everything(i):
        n, pages = inp.seq_lens.cpu().numpy(), inp.page_table.shape[1]
        used = -(-n // 16)
        shape = (4, step.levels[i], hkv)
        picks = np.broadcast_to(np.where(np.arange(pages) < used[:, None], np.arange(pages), -1)[:, None, None], (*shape, pages))
        return picks, np.broadcast_to(used[:, None, None], shape)
    # (draft_attn rounds P to bf16 too)
    check_levels(step, everything)
    assert w.error_code() == 0 and w.error_code() == 0


def test_a_captured_step_with_eviction_replays_as_it_runs():
    def steps():
        step.run()
        w.evict(300, 2, 16)
        step.run()
        w.evict(50, 2, 16)
    inp = inputs((3, 4), lens=(200, 130, 90, 700))
    w = TokenWeights(inp, decay=0.75)
    step = DraftStep(inp, weights=w)
    state = (inp.target_k, inp.target_v, inp.seq_lens, w.weights, w.free_pages, w.free_count)
    start = [x.clone() for x in state]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        steps()
    stream.synchronize()
    want = [x.clone() for x in (*state, *step.out, *step.lse)]
    assert inp.seq_lens.tolist() == [50, 50, 50, 50]
    for x, y in zip(state, start):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        steps()
    graph.replay()
    torch.cuda.synchronize()
    for x, y in zip((*state, *step.out, *step.lse), want):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    assert w.error_code() == 0 and step.error_code() == 0


def test_a_captured_step_over_selected_pages():
    inp = inputs((4, 4), lens=(900, 130, 90, 1200))
    step = DraftStep(inp, pages=PageSelection(inp, keep=9))
    step.run()
    torch.cuda.synchronize()
    want = [x.clone() for x in step.out]
    for x in step.out + step.lse:
        x.zero_()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        step.run()
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(step.out, want))
    check_levels(step, lambda i: picked(step, i))


def test_refusals():
    inp = inputs()
    pages, w = PageSelection(inp, keep=5), TokenWeights(inp)
    with pytest.raises(kvshot.KvshotError):
        PageSelection(inp, keep=4, first=3, last=2)
    with pytest.raises(kvshot.KvshotError):
        w.evict(10, 8, 3)
    with pytest.raises(ValueError):
        DraftStep(inp, pages=pages, weights=w)
    with pytest.raises(ValueError):
        DraftStep(inputs(), pages=pages)
    with pytest.raises(ValueError):
        DraftStep(inp, pages=pages, target_fp8=(None, None, 0, 0))
    spec = wl.Spec("contiguous", 1, 1, [30], [1], False, False, hq=8, hkv=2)
    with pytest.raises(ValueError):
        PageSelection(wl.make_inputs(spec, "cuda"), keep=5)
