"""The 4-bit cache as a drafting server uses it: pages found and tokens stored between steps, each step drafted over the
cache (append + attention at every drafting level), with and without a window, eagerly and from a captured graph.

Against the oracle's append and the 64-bit attention over the values that the cache holds.  Bounds as for the attention
alone (tests/test_gpu_kv4.py): the step adds no rounding of its own (the appended q and draft K/V are the oracle's bits).
"""
import numpy as np
import pytest
import torch

from oracle import kv4, oracle
from paper_2604_26412_gb300 import kv4 as user
from paper_2604_26412_gb300 import kvshot
from paper_2604_26412_gb300 import workloads as wl
from paper_2604_26412_gb300.step import DraftStep
from tests.test_gpu_kv4 import LSE_MAX_ABS, OUT_MAX_ABS, OUT_REL_L2

pytestmark = pytest.mark.gpu


def _inputs(levels, tree=True, layers=1, lens=(40, 0, 129), paged=True, seed=3):
    spec = wl.Spec("kv4-step", len(lens) // layers, layers, list(lens), levels, tree, paged, page_size=16, hq=8, hkv=2, seed=seed)
    return spec, wl.make_inputs(spec, "cuda", seed=seed, tail_fill="nan")


def _check(step, inp, cache):
    """Every level of the step against the oracle, over the cache's own values."""
    s = inp.spec
    dk = np.full((s.num_caches, s.hkv, inp.n_max, 128), 0x7FC0, np.uint16)
    dv = dk.copy()
    d = oracle.make_desc(num_caches=s.num_caches, num_seqs=s.num_seqs, hq=s.hq, hkv=s.hkv, head_dim=128, n_nodes=0,
                         n_query=0, n_max=inp.n_max, tree=s.tree, l_cap=1)
    lens = cache.seq_lens.cpu().numpy()
    table = cache.page_table.cpu().numpy()
    n0 = 0
    for i, n in enumerate(step.levels):
        q = oracle.append(d, wl.bf16_bits(step.q_in[i]), wl.bf16_bits(step.k_in[i]), wl.bf16_bits(step.v_in[i]),
                          step.pos[i].cpu().numpy(), n0, n, s.rope_base, dk, dv)
        n0 += n
        wide = lambda x: wl.bits_to_bf16(x).double().numpy()  # noqa: E731
        for c in range(s.num_caches):
            slots = [table[c, j // cache.page_size] * cache.page_size + j % cache.page_size for j in range(lens[c])]
            k, v = (x.double().cpu().numpy().swapaxes(0, 1)
                    for x in cache.values(torch.tensor(slots, dtype=torch.int32, device="cuda")))
            par = step.parents[i][c // s.layers].cpu().numpy() if s.tree else None
            out, lse = kv4.attn(wide(q[c]), k, v, wide(dk[c, :, :n0]), wide(dv[c, :, :n0]), par, step.window, step.sinks,
                                128 ** -0.5)
            o, l = step.out[i][c].double().cpu().numpy(), step.lse[i][c].double().cpu().numpy()
            assert np.abs(o - out).max() <= OUT_MAX_ABS, (i, c)
            assert np.linalg.norm(o - out) <= OUT_REL_L2 * np.linalg.norm(out), (i, c)
            assert np.abs(l - lse).max() <= LSE_MAX_ABS, (i, c)
    assert step.error_code() == 0 and cache.error_code() == 0


@pytest.mark.parametrize("mode", ["per_depth", "whole"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 5)])
@pytest.mark.parametrize("tree,layers,paged", [(True, 1, True), (False, 3, False)])
def test_steps_over_a_growing_cache(mode, window, sinks, tree, layers, paged):
    spec, inp = _inputs([2, 3] if tree else [1, 1, 1], tree, layers, paged=paged)
    cache = user.of_inputs(inp, spare_pages=6, spare_tokens=40)
    step = DraftStep(inp, mode=mode, target_kv4=cache, window=window, sinks=sinks)
    step.run()
    _check(step, inp, cache)
    want = sum(spec.seq_lens)
    for new in ([3, 1, 0], [0, 17, 8]):  # verified tokens; K and V as slices of wider rows
        t = sum(new)
        rows = torch.randn((t, spec.hkv * 3 * 128), device="cuda").to(torch.bfloat16)
        k = rows[:, :spec.hkv * 128].unflatten(1, (spec.hkv, 128))
        v = rows[:, spec.hkv * 256:].unflatten(1, (spec.hkv, 128))
        cache.grow(torch.tensor(new, dtype=torch.int32, device="cuda"), k, v)
        want += t
        got = cache.values(cache.slots[:t])[0].double().cpu().numpy()
        codes, scales = kv4.quantise(k.double().cpu().numpy(), 0)
        assert np.array_equal(got, kv4.values(codes, scales, 0))
        step.run()
        assert int(cache.seq_lens.sum()) == want
        _check(step, inp, cache)


def test_growth_and_step_from_a_graph():
    """Captured once, replayed twice: what two eager rounds give, bit for bit."""
    _, inp = _inputs([2, 3])
    new = torch.tensor([2, 5, 1], dtype=torch.int32, device="cuda")
    k, v = (torch.randn((8, 2, 128), device="cuda").to(torch.bfloat16) for _ in range(2))
    caches = [user.of_inputs(inp, spare_pages=8, spare_tokens=40) for _ in range(2)]
    steps = [DraftStep(inp, target_kv4=c, window=30, sinks=2) for c in caches]
    for _ in range(3):
        caches[0].grow(new, k, v)
        steps[0].run()
    caches[1].grow(new, k, v)  # (the first round, uncaptured)
    steps[1].run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caches[1].grow(new, k, v)
        steps[1].run()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(caches[0].seq_lens, caches[1].seq_lens) and torch.equal(caches[0].page_table, caches[1].page_table)
    for a, b in zip(steps[0].out, steps[1].out):
        assert torch.equal(a, b)
    _check(steps[1], inp, caches[1])


def test_a_pool_that_runs_out_takes_nothing():
    _, inp = _inputs([2])
    cache = user.of_inputs(inp, spare_pages=1, spare_tokens=40)
    before = cache.data.clone(), cache.seq_lens.clone()
    k = torch.ones((40, 2, 128), dtype=torch.bfloat16, device="cuda")
    cache.grow(torch.tensor([20, 0, 20], dtype=torch.int32, device="cuda"), k, k)
    assert cache.error_code() == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    assert torch.equal(before[0], cache.data) and torch.equal(before[1], cache.seq_lens)


def test_refusals():
    _, inp = _inputs([2])
    cache = user.of_inputs(inp)
    with pytest.raises(ValueError):
        DraftStep(inp, window=8)
    with pytest.raises(ValueError):
        DraftStep(inp, target_kv4=cache, target_fp8=(None, None, 0, 0))
    with pytest.raises(ValueError):
        DraftStep(inp, target_kv4=user.Kv4Cache(2, 2, 4, 4, max_tokens=8))
    k = torch.zeros((4, 2, 128), dtype=torch.bfloat16, device="cuda")
    for bad in (k.float(), k[:, :1], k.transpose(1, 2)):
        with pytest.raises(ValueError):
            cache.store(bad, bad)
    with pytest.raises(ValueError):
        cache.store(k, k, cache.slots[:3])
    with pytest.raises(kvshot.KvshotError):
        user.Kv4Cache(2, 2, 4, 4, page_size=8, max_tokens=8)


@pytest.mark.parametrize("hq,nodes,lens", [(8, 2, (3000, 517, 64)), (8, 4, (3000, 517, 64)), (8, 12, (3000, 517, 64)),
                                           (8, 40, (3000, 517, 64))])
def test_a_wait_that_runs_out_is_recorded(hq, nodes, lens):
    """8, 16, 48 and 160 rows with a limit of 1 ns: the call ends, records KVSHOT_ERR_TIMEOUT (or, where no wait was
    long enough, is right), and leaves everything fit for the next one."""
    from tests.test_gpu_kv4 import Case
    case = Case(list(lens), hq=hq, hkv=2, nodes=nodes, query=nodes, seed=nodes)
    want = case.run()
    for _ in range(3):
        case.desc.wait_limit_ns = 1
        case.run()
        assert int(case.err.item()) in (0, kvshot.KVSHOT_ERR_TIMEOUT)
        case.desc.wait_limit_ns = 0
        case.err.zero_()
        case.out.fill_(float("nan"))
        got = case.run()
        assert int(case.err.item()) == 0
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("lens,hq,nodes,num_ctas", [((3000,), 8, 2, 0), ((3000,), 8, 12, 7), ((700, 3000, 0, 150), 8, 4, 0),
                                                    ((2000, 1000), 8, 40, 3), ((9000,), 8, 1, 300), ((6000, 40), 8, 14, 120)])
def test_pieces_are_joined(lens, hq, nodes, num_ctas):
    """Units in one piece, in two and in more than 32, of one cache (cut by themselves) and of several."""
    from tests.test_gpu_kv4 import Case
    Case(list(lens), hq=hq, hkv=2, nodes=nodes, query=nodes, num_ctas=num_ctas, seed=nodes).check()


@pytest.mark.parametrize("nodes", [2, 4, 12])
def test_a_prefix_scale_that_underflows(nodes):
    """scale * 2^k_scale_exp below fp32: the prefix's scores are 0, its masked keys stay masked."""
    from tests.test_gpu_kv4 import Case
    Case([300], nodes=nodes, query=nodes, exps=(-64, 0), scale=1e-30, window=100, sinks=3, seed=nodes).check()


@pytest.mark.parametrize("window", [2 ** 31 - 1, 305, 304, 299])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("nodes", [2, 4, 12])
def test_windows_about_as_long_as_the_context(window, tree, nodes):
    from tests.test_gpu_kv4 import Case, _tree
    par = _tree(np.random.default_rng(nodes), 1, nodes, 2) if tree else None
    Case([300], nodes=nodes, query=nodes, parent=par, window=window, sinks=2, seed=nodes).check()


@pytest.mark.parametrize("lens", [(900, 1000, 900, 1000), (900, 10, 2500, 0)])
@pytest.mark.parametrize("nodes", [2, 4, 8, 12, 16])
@pytest.mark.parametrize("num_ctas", [8, 9, 16, 17, 23, 40])
def test_cuts(lens, nodes, num_ctas):
    """Eight units on as many CTAs and more: whole, cut by themselves (equal lengths), or laid end to end (unequal ones)."""
    from tests.test_gpu_kv4 import Case
    Case(list(lens), hq=8, hkv=2, nodes=nodes, query=nodes, num_ctas=num_ctas, seed=nodes).check()


@pytest.mark.parametrize("lens", [[0] * 40, [0, 3] * 20, [0, 130, 0, 0, 0, 1] * 7])
@pytest.mark.parametrize("nodes,hq", [(12, 8), (33, 8), (2, 8), (40, 8), (9, 8)])
@pytest.mark.parametrize("num_ctas", [1, 3])
def test_many_short_pieces_to_a_cta(lens, nodes, hq, num_ctas):
    """Pieces of one or two tiles, each of another tree: what a piece's end still reads must outlast the next ones' starts."""
    from tests.test_gpu_kv4 import Case, _tree
    par = _tree(np.random.default_rng(nodes), len(lens), nodes, 3)
    case = Case(list(lens), hq=hq, hkv=2, nodes=nodes, query=nodes, parent=par, num_ctas=num_ctas, seed=nodes)
    case.check(caches=range(0, len(lens), 3))
    first = case.run()
    for _ in range(5):
        again = case.run()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("counts", [[2 ** 30] * 4, [2 ** 30] * 2, [2 ** 31 - 1, 1], [1, 0, 2 ** 30 + 5] * 300])
def test_an_extension_beyond_32_bits_takes_nothing(counts):
    """Token counts whose sums pass 2^31 and 2^32."""
    c, page = len(counts), 1 << 20
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lens, new, free, count = i32([0] * c), i32(counts), i32(list(range(2000))), i32([2000])
    table = i32(np.full((c, 2047), 7).tolist())
    start, maps, err = i32([-5] * (c + 1)), [i32([0] * 64) for _ in range(3)], i32([0])
    desc = kvshot.make_extend_desc(num_caches=c, page_size=page, max_pages_per_seq=2047, num_pages=2000, max_tokens=64,
                                   err_flag=err)
    kvshot.cache_extend(desc, lens, new, table, free, count, lens, table, count, start, *maps)
    assert int(err.item()) == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    assert int(lens.abs().max()) == 0 and int(count.item()) == 2000 and bool((table == 7).all())
    assert int(start.abs().max()) == 0 and all(bool((m == -1).all()) for m in maps)
