"""Calls that draft over a part of a long cache on another stream, captured in a graph, beside one another, and with waits that
run out: the kernels that large calls take among them."""
import numpy as np
import pytest
import torch

from oracle import partial
from paper_2604_26412_gb300 import kvshot

from .partial_problems import D, Problem, f64
from .test_gpu_partial import MANY, SHARED, check, run_scores, run_sparse, run_weights, some_lse

pytestmark = pytest.mark.gpu


def calls(p, keep=9, seed=0):
    """One of each call over p's caches; returns (run(stream), outputs)."""
    c, pages = len(p.lens), p.table.shape[1]
    picks, counts = p.random_picks(keep, seed=seed)
    dev = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    o = {"bounds": dev(p.num_pages, p.hkv, 2, D, dtype=torch.bfloat16), "scores": dev(c, p.Nq, p.hkv, pages),
         "picks": dev(c * p.Nq * p.hkv, keep, dtype=torch.int32), "counts": dev(c * p.Nq * p.hkv, dtype=torch.int32),
         "out": torch.zeros_like(p.q), "lse": dev(c, p.Nq, p.hq), "weights": dev(c, int(p.lens.max()) + 1),
         "tokens": dev(c, 50, dtype=torch.int32), "kept": dev(c, dtype=torch.int32)}
    sel = kvshot.make_select_desc(num_rows=c * p.Nq * p.hkv, row_len=pages, rows_per_len=p.Nq * p.hkv,
                                  tokens_per_entry=p.page, keep=keep, first=1, last=2, err_flag=p.err)
    tok = kvshot.make_select_desc(num_rows=c, row_len=o["weights"].shape[1], keep=50, first=4, last=8, err_flag=p.err)
    given, n, lse = p.ints(picks), p.ints(counts), torch.from_numpy(some_lse(p)).cuda()
    ws = p.workspace(keep)

    def run(stream=None):
        kvshot.page_bounds(p.desc, p.k, p.t_table, p.t_lens, None, o["bounds"], stream)
        kvshot.page_scores(p.desc, p.q, o["bounds"], p.t_table, p.t_lens, o["scores"], stream)
        kvshot.select_top(sel, o["scores"], p.t_lens, o["picks"], o["counts"], stream)
        kvshot.draft_attn_sparse(p.desc, p.q, p.k, p.v, p.t_table, p.t_lens, given, n, keep, p.dk, p.dv, p.t_parent, o["out"],
                                 o["lse"], stream)
        kvshot.key_weights(p.desc, p.q, p.k, p.t_table, p.t_lens, lse, 0.5, o["weights"].shape[1], o["weights"], o["weights"],
                           stream)
        kvshot.select_top(tok, o["weights"], p.t_lens, o["tokens"], o["kept"], stream)
    run.keep_alive = (ws, given, n, lse)
    return run, o


def large():
    """Shared pages in the sparse attention, tcgen05 for the weights, a cluster for each cache's tokens."""
    return Problem([300, 9001, 700, 64, 65, 128, 500, 33, 31, 900, 1000, 77, 90], 16, nodes=12, query=12, tree=True, seed=3)


@pytest.mark.parametrize("make", [large, lambda: Problem([300, 0, 65], 16, nodes=3, query=2, seed=5),
                                  lambda: Problem(**MANY["level"], seed=6)])
def test_other_streams_and_graphs_give_the_same(make):
    p = make()
    run, o = calls(p)
    run()
    check(p)
    want = {k: v.clone() for k, v in o.items()}

    def again(f):
        for v in o.values():
            v.zero_()
        torch.cuda.synchronize()
        f()
        torch.cuda.synchronize()
        for k in o:
            assert torch.equal(o[k].view(torch.int16), want[k].view(torch.int16)), k
        assert int(p.err.item()) == 0
    stream = torch.cuda.Stream()
    again(lambda: run(stream))
    with torch.cuda.stream(stream):
        again(run)
    graph = torch.cuda.CUDAGraph()
    for v in o.values():
        v.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        run()
    again(graph.replay)
    again(graph.replay)


def test_two_calls_at_once():
    a, b = large(), large()
    b.q *= 0.5
    b.k *= 0.5
    runs = [calls(a), calls(b)]
    want = []
    for run, o in runs:
        run()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in o.items()})
        for v in o.values():
            v.zero_()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for (run, _), s in zip(runs, streams):
        run(s)
    torch.cuda.synchronize()
    for (_, o), w in zip(runs, want):
        for k in o:
            assert torch.equal(o[k].view(torch.int16), w[k].view(torch.int16)), k


def test_waits_that_run_out_are_reported_and_the_next_calls_are_right():
    p = Problem(**SHARED["tree"], seed=2)
    picks, counts = p.random_picks(9)
    w = Problem([700, 300, 65], 16, nodes=24, query=24, seed=3)
    m = Problem(**MANY["level"], seed=4)
    bounds = torch.randn((m.num_pages, 8, 2, D), device="cuda").sort(dim=2).values.to(torch.bfloat16)
    for _ in range(2):  # (twice in a row: a call that gave up leaves nothing that blocks the next one)
        p.desc.wait_limit_ns = w.desc.wait_limit_ns = m.desc.wait_limit_ns = 1
        ws = p.workspace(9)
        kvshot.draft_attn_sparse(p.desc, p.q, p.k, p.v, p.t_table, p.t_lens, p.ints(picks), p.ints(counts), 9, p.dk, p.dv,
                                 p.t_parent, torch.empty_like(p.q), torch.empty(p.q.shape[:3], device="cuda"))
        check(p, kvshot.KVSHOT_ERR_TIMEOUT)
        kvshot.key_weights(w.desc, w.q, w.k, w.t_table, w.t_lens, torch.from_numpy(some_lse(w)).cuda(), 0.0, 700, None,
                           torch.empty((3, 700), device="cuda"))
        check(w, kvshot.KVSHOT_ERR_TIMEOUT)
        kvshot.page_scores(m.desc, m.q, bounds, m.t_table, m.t_lens, torch.empty((40, 12, 8, m.table.shape[1]), device="cuda"))
        check(m, kvshot.KVSHOT_ERR_TIMEOUT)
        m.err.zero_()
        p.err.zero_()
        w.err.zero_()
        del ws
    p.desc.wait_limit_ns = w.desc.wait_limit_ns = m.desc.wait_limit_ns = 0
    run_sparse(p, picks, counts)
    run_weights(w)
    run_scores(m, bounds)


def test_weights_do_not_change_from_run_to_run():
    p = Problem([700, 1300, 65], 16, nodes=64, query=64, seed=4)
    a, b = run_weights(p, given=False), run_weights(p, given=False)
    assert torch.equal(a, b)


def test_an_eviction_reads_what_an_extension_wrote():
    """Pages go round: tokens evicted, their pages given back, and taken again by the next tokens."""
    p = Problem([100, 60], 16, hq=2, hkv=2, seed=6)
    pool = p.num_pages
    free = torch.full((pool,), -1, dtype=torch.int32, device="cuda")
    count = p.ints([0])
    lens, table = p.t_lens.clone(), p.t_table.clone()
    w = torch.arange(2 * 128, dtype=torch.float32, device="cuda").reshape(2, 128)
    sel = kvshot.make_select_desc(num_rows=2, row_len=128, keep=33, err_flag=p.err)
    kept, n = torch.zeros((2, 33), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ev = kvshot.make_evict_desc(num_caches=2, hkv=2, page_size=16, max_pages_per_seq=table.shape[1], num_pages=pool,
                                max_kept=33, weights_len=128, err_flag=p.err)
    ext = kvshot.make_extend_desc(num_caches=2, page_size=16, max_pages_per_seq=table.shape[1], num_pages=pool, max_tokens=64,
                                  err_flag=p.err)
    slots = [torch.zeros(64, dtype=torch.int32, device="cuda") for _ in range(3)]
    start = torch.zeros(3, dtype=torch.int32, device="cuda")
    before = table.cpu().numpy().copy()
    kvshot.select_top(sel, w, lens, kept, n)
    kvshot.cache_evict(ev, p.k, p.v, table, lens, kept, n, w, p.k, p.v, table, lens, w, free, count, count)
    kvshot.cache_extend(ext, lens, p.ints([30, 20]), table, free, count, lens, table, count, start, *slots)
    check(p)
    assert lens.tolist() == [63, 53]
    given = [int(x) for c, lo, hi in ((0, 3, 7), (1, 3, 4)) for x in before[c, lo:hi]]
    got = table.cpu().numpy()
    assert sorted([got[0, 3], got[1, 3]]) == sorted(given[-2:]) and int(count.item()) == len(given) - 2
    assert np.array_equal(got[:, :3], before[:, :3])
    assert torch.equal(w[0, :33], torch.arange(67, 100, dtype=torch.float32, device="cuda")) and float(w[:, 33:].abs().max()) == 0
