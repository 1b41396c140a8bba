"""Drafting over a part of a long cache on the GPU against the fp64 oracle.

Tolerances.  A sum of n products on the tensor cores is fp32; every addition is off by at most a step, 2^-23, of the sum of
the products' magnitudes S, so a dot product over 128 dims (256 for the scores) by at most 2^-16 S (2^-15 S).
  scores   2^-15 S
  weights  every term's exponent is off by 2^-16 (S + |lse|) + 2^-22 of the exponential itself, and the sum of T terms by
           T 2^-24, all relative to the value
  lse      2^-16 S + 2^-18 (exponentials, sums and logarithm)
  out      P and the result are rounded to bf16, 2^-8 each, relative to sum p |v|; and the error of lse
Everything else is exact.
"""
import numpy as np
import pytest
import torch

from oracle import partial
from paper_2604_26412_gb300 import kvshot

from .partial_problems import D, Problem, f64

pytestmark = pytest.mark.gpu

LENS = [0, 1, 7, 8, 9, 63, 64, 65, 130, 257, 300]


def check(p, code=0):
    torch.cuda.synchronize()
    assert int(p.err.item()) == code


# ------------------------------------------------------------ bounds

@pytest.mark.parametrize("page", [8, 16, 64, 192, 256])
@pytest.mark.parametrize("hkv", [1, 8, 3])
def test_bounds(page, hkv):
    p = Problem(LENS, page, hq=hkv, hkv=hkv, seed=page)
    out = torch.full((p.num_pages, hkv, 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
    want = partial.page_bounds(f64(p.k), p.table, p.lens, np.zeros(len(LENS)), f64(out))
    kvshot.page_bounds(p.desc, p.k, p.t_table, p.t_lens, None, out)
    check(p)
    assert np.array_equal(f64(out), want)


@pytest.mark.parametrize("new", [0, 1, 16, 17, 1000])
def test_bounds_of_new_tokens_alone(new):
    p = Problem(LENS, 16, seed=new)
    before = np.maximum(0, p.lens - new)
    out = torch.full((p.num_pages, 8, 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
    want = partial.page_bounds(f64(p.k), p.table, p.lens, before, f64(out))
    kvshot.page_bounds(p.desc, p.k, p.t_table, p.t_lens, p.ints(before), out)
    check(p)
    assert np.array_equal(f64(out), want)


def test_bounds_of_nan_and_infinities():
    p = Problem([40], 16)
    p.k[p.table[0, 0], 2, 5, 9] = float("nan")
    p.k[p.table[0, 1], 3, 0, 0] = float("inf")
    p.k[p.table[0, 1], 3, 1, 0] = float("-inf")
    out = torch.zeros((p.num_pages, 8, 2, D), dtype=torch.bfloat16, device="cuda")
    want = partial.page_bounds(f64(p.k), p.table, p.lens, [0], f64(out))
    kvshot.page_bounds(p.desc, p.k, p.t_table, p.t_lens, None, out)
    check(p)
    assert np.array_equal(f64(out), want, equal_nan=True)
    assert np.isnan(want).sum() == 2


# ------------------------------------------------------------ scores

def run_scores(p, bounds):
    out = torch.full((len(p.lens), p.Nq, p.hkv, p.table.shape[1]), 7.0, device="cuda")
    want, mag = partial.page_scores(f64(p.q), f64(bounds), p.table, p.lens, p.page, p.scale, f64(out))
    kvshot.page_scores(p.desc, p.q, bounds, p.t_table, p.t_lens, out)
    check(p)
    assert np.all(np.abs(f64(out) - want) <= 2.0 ** -15 * mag + 2.0 ** -23 * np.abs(want))
    return f64(out)


@pytest.mark.parametrize("hq,hkv", [(32, 8), (8, 8), (16, 8), (28, 4), (12, 4), (8, 1), (16, 1), (32, 1), (40, 2), (9, 1)])
@pytest.mark.parametrize("query", [1, 5, 33])
def test_scores(hq, hkv, query):
    p = Problem([0, 1, 15, 16, 17, 700], 8, hq=hq, hkv=hkv, nodes=query, query=query, seed=hq + query)
    b = torch.randn((p.num_pages, hkv, 2, D), device="cuda").sort(dim=2).values.to(torch.bfloat16)
    run_scores(p, b)


def test_scores_of_a_call_of_many_pages_bound_every_key():
    p = Problem([5003], 16, nodes=3, query=3, scale=0.3)
    b = torch.zeros((p.num_pages, 8, 2, D), dtype=torch.bfloat16, device="cuda")
    kvshot.page_bounds(p.desc, p.k, p.t_table, p.t_lens, None, b)
    got = run_scores(p, b)
    for h in range(8):
        rows = partial.rows_of(f64(p.k), p.table, 0, 5003, h)
        s = 0.3 * np.einsum("ngd,jd->ngj", f64(p.q)[0, :, 4 * h:4 * h + 4], rows).max(1)
        assert np.all(got[0, :, h].repeat(16, axis=-1)[:, :5003] >= s - 1e-4)


MANY = {  # calls of 48 rows per KV head and more over many tiles of 128 pages
    "level": dict(lens=[0, 1, 8, 1016, 1023, 1024, 1025, 1032, 2049, 5003] * 4, page=8, nodes=12, query=12),
    "one head": dict(lens=[40] * 20 + [2100] * 40, page=16, hq=8, hkv=8, nodes=70, query=70),
    "pairs": dict(lens=[0] * 40 + [1030] * 80, page=8, hq=16, hkv=8, nodes=33, query=33),
    "seven heads": dict(lens=list(range(0, 1600, 16)), page=8, hq=28, hkv=4, nodes=9, query=9),
    "14 heads": dict(lens=[1030] * 20, page=8, hq=112, hkv=8, nodes=8, query=8),
    "17 heads": dict(lens=[1100] * 40, page=8, hq=34, hkv=2, nodes=5, query=5),
    "one KV head": dict(lens=[1100] * 200, page=8, hq=32, hkv=1, nodes=4, query=4),
    "whole tree": dict(lens=[33000, 0, 200], page=8, nodes=64, query=64),
}


@pytest.mark.parametrize("name", MANY)
def test_scores_of_many_pages(name):
    p = Problem(**MANY[name], seed=len(name))
    b = torch.randn((p.num_pages, p.hkv, 2, D), device="cuda").sort(dim=2).values.to(torch.bfloat16)
    first = run_scores(p, b)
    assert np.array_equal(first, run_scores(p, b))


def test_scores_of_many_pages_pass_over_bad_pages_and_lengths():
    p = Problem(**MANY["level"], seed=1)
    b = torch.randn((p.num_pages, 8, 2, D), device="cuda").sort(dim=2).values.to(torch.bfloat16)
    good = torch.full((40, 12, 8, p.table.shape[1]), 7.0, device="cuda")
    kvshot.page_scores(p.desc, p.q, b, p.t_table, p.t_lens, good)
    check(p)
    for at, bad in (((9, 3), p.num_pages), ((19, 200), -1), ((28, 128), 2 ** 31 - 1)):
        table, want = p.t_table.clone(), good.clone()
        table[at], want[at[0], :, :, at[1]] = bad, 7.0
        got = torch.full_like(good, 7.0)
        kvshot.page_scores(p.desc, p.q, b, table, p.t_lens, got)
        check(p, kvshot.KVSHOT_ERR_DEVICE_BOUNDS)
        assert torch.equal(got, want)
        p.err.zero_()
    lens, want, got = p.t_lens.clone(), good.clone(), torch.full_like(good, 7.0)
    lens[9], want[9] = -5, 7.0
    kvshot.page_scores(p.desc, p.q, b, p.t_table, lens, got)
    check(p, kvshot.KVSHOT_ERR_DEVICE_BOUNDS)
    assert torch.equal(got, want)


# ------------------------------------------------------------ selection

def run_select(scores, lens, per, unit, keep, first, last, code=0):
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    s = torch.from_numpy(np.ascontiguousarray(scores, dtype=np.float32)).cuda()
    picks = torch.full((len(scores), keep), 99, dtype=torch.int32, device="cuda")
    counts = torch.full((len(scores),), 99, dtype=torch.int32, device="cuda")
    d = kvshot.make_select_desc(num_rows=len(scores), row_len=s.shape[1], rows_per_len=per, tokens_per_entry=unit, keep=keep,
                                first=first, last=last, err_flag=err)
    kvshot.select_top(d, s, torch.tensor(np.asarray(lens), dtype=torch.int32, device="cuda"), picks, counts)
    torch.cuda.synchronize()
    assert int(err.item()) == code
    want, n = partial.select_top(s.cpu().numpy().astype(np.float64), lens, per, unit, keep, first, last)
    assert np.array_equal(counts.cpu().numpy(), n)
    assert np.array_equal(picks.cpu().numpy(), want)


def some_scores(kind, rows, n, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, n))
    if kind == "ties":
        return np.round(x * 2) / 2 * np.where(rng.random(x.shape) < 0.5, 1.0, -1.0)  # (-0 among them)
    if kind == "equal":
        return np.full((rows, n), -1.5)
    if kind == "close":
        return 1 + np.round(np.abs(x) * 8) * 2.0 ** -23
    if kind == "special":
        for v in (np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-42, -1e-42):
            x[rng.random(x.shape) < 0.1] = v
    if kind == "weights":
        return np.exp(4 * x)
    return x


@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "close", "special", "weights"])
@pytest.mark.parametrize("n,keep,first,last", [(1, 1, 0, 0), (33, 1, 0, 0), (64, 64, 3, 5), (100, 64, 3, 5), (700, 699, 0, 1),
                                               (700, 60, 20, 40), (2049, 128, 1, 4), (5000, 1024, 0, 512)])
def test_select(kind, n, keep, first, last):
    run_select(some_scores(kind, 3, n, n + keep), [n, max(1, n - 13), n], 1, 1, keep, first, last)


@pytest.mark.parametrize("n", [20011, 60000, 131072, 300001])
def test_select_of_long_rows(n):
    for kind, keep in (("weights", 4096), ("close", n // 2), ("special", 17)):
        run_select(some_scores(kind, 2, n, n), [n, n - 1000], 1, 1, keep, 16 if keep > 100 else 0, keep // 8)


@pytest.mark.parametrize("n,keep", [(700, 60), (5000, 600), (20000, 2000), (150000, 9)])
def test_select_takes_every_nan_alike(n, keep):
    """NaNs of either sign and of any payload come first, in their entries' order; every -inf last but two zeros alike."""
    x = np.where(np.arange(2 * n).reshape(2, n) % 5 == 0, 0.0, -np.inf).astype(np.float32)
    bits = x.view(np.uint32)
    bits[0, ::n // 40] = 0xff800001  # (a signalling one, negative)
    bits[0, 7::n // 40] = 0x7fffffff
    bits[1, 3::n // 30] = 0xffc00000
    bits[1, ::10] = 0x80000000
    run_select(x, [n, n - 1], 1, 1, keep, 1, 2)


def test_select_of_the_pages_of_ragged_caches():
    lens = [0, 1, 16, 17, 1000, 555]
    run_select(some_scores("ties", len(lens) * 24, 63, 3), lens, 24, 16, 12, 1, 2)


def test_select_records_lengths_out_of_range():
    s = some_scores("normal", 3, 40, 1)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    picks, counts = torch.zeros((3, 8), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    d = kvshot.make_select_desc(num_rows=3, row_len=40, keep=8, err_flag=err)
    kvshot.select_top(d, torch.from_numpy(s).float().cuda(), torch.tensor([-3, 2 ** 31 - 1, 12], dtype=torch.int32, device="cuda"),
                      picks, counts)
    torch.cuda.synchronize()
    assert int(err.item()) == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    want, n = partial.select_top(s.astype(np.float32).astype(np.float64), [0, 40, 12], 1, 1, 8, 0, 0)
    assert np.array_equal(picks.cpu().numpy(), want) and np.array_equal(counts.cpu().numpy(), n)


# ------------------------------------------------------------ sparse attention

def run_sparse(p, picks, counts, code=0, kept=None):
    keep = picks.shape[-1]
    ws = p.workspace(keep)
    out, lse = torch.full_like(p.q, 7.0), torch.full(p.q.shape[:3], 7.0, device="cuda")
    kvshot.draft_attn_sparse(p.desc, p.q, p.k, p.v, p.t_table, p.t_lens, p.ints(picks), p.ints(counts), keep, p.dk, p.dv,
                             p.t_parent, out, lse)
    check(p, code)
    del ws
    if kept is not None:
        picks, counts = kept
    want, z, spread, mag = partial.attn_sparse(f64(p.q), f64(p.k), f64(p.v), p.table, p.lens, picks, counts, f64(p.dk),
                                               f64(p.dv), p.parent, p.layers, p.N, p.scale)
    tol_z = 2.0 ** -16 * mag + 2.0 ** -18
    assert np.all(np.abs(f64(lse) - z) <= tol_z)
    assert np.all(np.abs(f64(out) - want) <= (2.0 ** -7 + 2 * tol_z[..., None]) * spread)
    return out, lse


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 192, 256])
@pytest.mark.parametrize("nodes,query,tree", [(1, 1, False), (9, 4, False), (30, 7, True)])
def test_sparse_pages(page, nodes, query, tree):
    p = Problem([0, 1, 8, 100, 513, 700], page, nodes=nodes, query=query, tree=tree, layers=2, seed=page)
    run_sparse(p, *p.random_picks(6, seed=page))


@pytest.mark.parametrize("hq,hkv", [(8, 8), (16, 8), (28, 4), (8, 1), (12, 1), (16, 1), (32, 1), (34, 2), (9, 1), (64, 2)])
def test_sparse_heads(hq, hkv):
    p = Problem([3, 333, 90], 16, hq=hq, hkv=hkv, nodes=12, query=5, tree=True, seed=hq)
    run_sparse(p, *p.random_picks(9, seed=hq))


@pytest.mark.parametrize("lens,keep,query", [([9000], 500, 1), ([9000], 3, 1), ([4100, 37], 257, 2), ([300] * 40, 19, 8)])
def test_sparse_lists_of_every_length(lens, keep, query):
    p = Problem(lens, 16, nodes=query, query=query, seed=keep)
    run_sparse(p, *p.random_picks(keep, seed=keep))


def test_sparse_without_any_page_attends_to_the_draft_alone():
    p = Problem([100, 0], 16, nodes=4, query=4)
    picks, counts = np.full((2, 4, 8, 5), -1, np.int32), np.zeros((2, 4, 8), np.int32)
    out, _ = run_sparse(p, picks, counts)
    first = p.dv[:, :, 0].repeat_interleave(4, dim=1)  # the first node sees itself alone
    assert torch.equal(out[:, 0], first)


@pytest.mark.parametrize("nodes", [65, 100, 200])
def test_sparse_long_chains(nodes):
    p = Problem([50, 333], 64, nodes=nodes, query=3, seed=nodes)
    run_sparse(p, *p.random_picks(4, seed=nodes))


def test_sparse_a_tree_of_64_in_a_line():
    p = Problem([50], 16, nodes=64, query=2, tree=True)
    p.parent = np.arange(-1, 63, dtype=np.int32)[None]
    p.t_parent = p.ints(p.parent)
    run_sparse(p, *p.random_picks(2))


def test_sparse_pages_that_are_not_picked_are_not_read():
    p = Problem([900], 16, nodes=2, query=2)
    picks, counts = p.random_picks(7, seed=5)
    seen = {int(x) for x in picks.reshape(-1) if x >= 0}
    for i in range(-(-900 // 16)):
        if i not in seen:
            p.k[p.table[0, i]] = float("nan")
            p.v[p.table[0, i]] = float("nan")
            p.t_table[0, i] = -5
    run_sparse(p, picks, counts)


@pytest.mark.parametrize("scale,std", [(1.0, 4.0), (0.05, 0.5), (3.0, 8.0)])
def test_sparse_scales(scale, std):
    p = Problem([700, 40], 32, nodes=3, query=3, scale=scale, std=std, seed=11)
    run_sparse(p, *p.random_picks(20, seed=2))


def test_sparse_a_rising_line_of_scores_moves_the_reference():
    p = Problem([512], 16, nodes=1, query=1)
    ramp = torch.linspace(-40, 40, 512).to(torch.bfloat16).cuda()
    p.q[:] = 0
    p.q[..., 0] = 8
    for i in range(32):
        p.k[p.table[0, i], :, :, 0] = ramp[16 * i:16 * i + 16]
    picks = np.broadcast_to(np.arange(32, dtype=np.int32), (1, 1, 8, 32))
    run_sparse(p, picks, np.full((1, 1, 8), 32, np.int32))


def test_sparse_all_pages_agree_with_draft_attention():
    p = Problem([700, 64, 1], 16, nodes=10, query=10, tree=True, seed=4)
    picks = np.full((3, 10, 8, 44), -1, np.int32)
    counts = np.zeros((3, 10, 8), np.int32)
    for c, n in enumerate(p.lens):
        m = -(-int(n) // 16)
        picks[c, :, :, :m], counts[c] = np.arange(m), m
    out, lse = run_sparse(p, picks, counts)
    table = p.t_table.clamp(min=0)
    size = kvshot.workspace_size(p.desc)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    p.desc.workspace, p.desc.workspace_bytes = ws.data_ptr(), size
    full, z = torch.empty_like(out), torch.empty_like(lse)
    kvshot.draft_attn(p.desc, p.q, p.k, p.v, table, p.t_lens, p.dk, p.dv, p.t_parent, full, z)
    check(p)
    assert (full.float() - out.float()).abs().max() <= 0.03 and (z - lse).abs().max() <= 1e-3


# Calls whose nodes share pages: 32 rows per KV head and more that pick 128 tokens or more each, over two thirds of the SMs' number
# of (cache, head, 64 rows).
SHARED = {
    "tree": dict(lens=[0, 1, 15, 16, 17, 300, 700, 64, 65, 128, 500, 33, 8, 9], page=16, nodes=30, query=8, tree=True, layers=2),
    "chain": dict(lens=[0, 1, 7, 8, 9, 300, 700, 64, 65, 128, 500, 33, 31], page=8, nodes=20, query=16),
    "seven heads": dict(lens=list(range(0, 520, 20)), page=64, hq=28, hkv=4, nodes=6, query=5),
    "one KV head": dict(lens=list(range(51)) + [130], page=32, hq=32, hkv=1, nodes=4, query=4),
    "17 heads": dict(lens=list(range(0, 260, 10)), page=128, hq=34, hkv=2, nodes=3, query=3),
    "one head": dict(lens=list(range(0, 390, 30)), page=16, hq=8, hkv=8, nodes=64, query=64, tree=True),
    "whole tree": dict(lens=[200, 1000, 0, 191], page=192, nodes=64, query=64, tree=True),
    "long chain": dict(lens=list(range(0, 1300, 100)), page=256, nodes=100, query=12),
    "two windows": dict(lens=[20001, 9000] + [30] * 11, page=8, nodes=8, query=8),
    "65 rows": dict(lens=[177] * 7, page=16, hq=8, hkv=8, nodes=65, query=65),
}


@pytest.mark.parametrize("name", SHARED)
def test_sparse_shared_pages(name):
    p = Problem(**SHARED[name], seed=len(name))
    run_sparse(p, *p.random_picks(40 if name == "two windows" else 16, seed=len(name)))


def test_sparse_shared_pages_without_picks_and_bit_for_bit():
    p = Problem(**SHARED["tree"], seed=1)
    picks, counts = p.random_picks(9)
    counts[:, ::2] = 0
    counts[3] = 0
    a, b = run_sparse(p, picks, counts), run_sparse(p, picks, counts)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("scale,std", [(1.0, 4.0), (0.05, 0.5), (3.0, 8.0)])
def test_sparse_shared_scales(scale, std):
    p = Problem(**SHARED["chain"], scale=scale, std=std, seed=12)
    run_sparse(p, *p.random_picks(16, seed=12))


def test_sparse_shared_scores_that_rise_and_fall_along_the_cache():
    """Keys of every tile longer than the last one's, then shorter again, and rows whose scores all fall: references that move
    at each tile, beside rows that keep theirs."""
    p = Problem([1500] * 13, 16, nodes=8, query=8, std=2.0, seed=13)
    for i, row in enumerate(p.table):
        for at, page in enumerate(row[:94]):
            p.k[page] *= float(1 + (at // 8 if i % 2 else 12 - at // 8))
    p.q[:, 3] = -p.q[:, 2].abs()
    picks = np.broadcast_to(np.arange(94, dtype=np.int32), (13, 8, 8, 94))
    run_sparse(p, picks, np.full((13, 8, 8), 94, np.int32))


def test_sparse_shared_bad_picks_pages_and_parents():
    p = Problem([100] * 12 + [150], 16, nodes=8, query=8, tree=True)
    picks = np.full((13, 8, 8, 8), -1, np.int32)
    picks[..., :3] = [1, 3, 6]
    n = np.full((13, 8, 8), 3, np.int32)
    for row in ([1, 3, 6, 7, 2 ** 31 - 1, -1], [-9, -2, 1, 3, 3, 6], [1, 3, 6, 6, 6, -2 ** 31]):
        bad, counts = picks.copy(), n.copy()
        bad[4, 7, 2, :6], counts[4, 7, 2] = row, 6
        run_sparse(p, bad, counts, kvshot.KVSHOT_ERR_DEVICE_BOUNDS, (picks, n))
        p.err.zero_()
    full, many = picks.copy(), n.copy()
    full[5], many[5] = np.arange(8), 2 ** 30  # (of which 7 are pages)
    want, seven = full.copy(), n.copy()
    seven[5] = 7
    run_sparse(p, full, many, kvshot.KVSHOT_ERR_DEVICE_BOUNDS, (want, seven))
    p.err.zero_()
    for parents, table, code in (([-1, 0, 5, 1, 2, 3, 4, 5], p.t_table, kvshot.KVSHOT_ERR_TREE),
                                 ([-1, 0, 1, 1, 2, 3, 4, 5], p.t_table - p.num_pages, kvshot.KVSHOT_ERR_DEVICE_BOUNDS)):
        ws = p.workspace(8)
        kvshot.draft_attn_sparse(p.desc, p.q, p.k, p.v, table, p.t_lens, p.ints(picks), p.ints(n), 8, p.dk, p.dv,
                                 p.ints([parents] * 13), torch.empty_like(p.q), torch.empty(p.q.shape[:3], device="cuda"))
        check(p, code)
        p.err.zero_()
        del ws


@pytest.mark.parametrize("query", [1, 3])
def test_sparse_bad_picks_are_recorded(query):
    p = Problem([100], 16, nodes=query, query=query)
    good = np.full((1, query, 8, 6), -1, np.int32)
    good[..., :3] = [1, 3, 6]
    n = np.full((1, query, 8), 3, np.int32)
    for row, times in (([1, 3, 6, 7, 2 ** 31 - 1, -1], 6), ([-9, -2, 1, 3, 3, 6], 6), ([1, 1, 3, 3, 6, 6], 6),
                       ([1, 3, 6, 6, 6, -2 ** 31], 6)):  # (what is not a pick is passed over: the same three pages are left)
        bad = good.copy()
        bad[0, query - 1, 2] = row
        counts = n.copy()
        counts[0, query - 1, 2] = times
        run_sparse(p, bad, counts, kvshot.KVSHOT_ERR_DEVICE_BOUNDS, (good, n))
        p.err.zero_()
    run_sparse(p, np.ascontiguousarray(good[..., :3]), np.full((1, query, 8), 2 ** 30, np.int32), kvshot.KVSHOT_ERR_DEVICE_BOUNDS, (good, n))
    p.err.zero_()
    run_sparse(p, good, np.full((1, query, 8), -1, np.int32), kvshot.KVSHOT_ERR_DEVICE_BOUNDS, (good, 0 * n))


@pytest.mark.parametrize("query", [1, 5])
def test_sparse_bad_parents_and_pages_are_recorded(query):
    p = Problem([100], 16, nodes=5, query=query, tree=True)
    picks, counts = p.random_picks(4)
    args = (p.dk, p.dv)
    for parents, table, code in (([-1, 0, 5, 1, 2], p.t_table, kvshot.KVSHOT_ERR_TREE), ([-1, 0, -2, 1, 2], p.t_table, kvshot.KVSHOT_ERR_TREE),
                                 ([-1, 0, 1, 1, 2], p.t_table + p.num_pages, kvshot.KVSHOT_ERR_DEVICE_BOUNDS)):
        ws = p.workspace(4)
        kvshot.draft_attn_sparse(p.desc, p.q, p.k, p.v, table, p.t_lens, p.ints(picks), p.ints(counts), 4, *args,
                                 p.ints([parents]), torch.empty_like(p.q), torch.empty(p.q.shape[:3], device="cuda"))
        check(p, code)
        p.err.zero_()
        del ws


def test_sparse_runs_repeat_bit_for_bit():
    p = Problem([3000, 777], 16, nodes=4, query=4, seed=9)
    picks, counts = p.random_picks(64, seed=1)
    a, b = run_sparse(p, picks, counts), run_sparse(p, picks, counts)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------ weights

def some_lse(p, seed=0):
    """lse as a softmax over the prefix and more would have it."""
    C, Nq, hq = p.q.shape[:3]
    z = np.zeros((C, Nq, hq))
    k, q = f64(p.k), f64(p.q)
    for c in range(C):
        for head in range(hq):
            rows = partial.rows_of(k, p.table if p.t_table is not None else None, c, int(p.lens[c]), head // (hq // p.hkv))
            s = p.scale * (q[c, :, head] @ rows.T)
            z[c, :, head] = np.log(1 + np.exp(s).sum(-1))
    return z.astype(np.float32)


def run_weights(p, decay=1.0, given=True, lse=None, width=None, alias=False, code=0):
    width = width or max(1, int(p.lens.max())) + 2
    lse = some_lse(p) if lse is None else lse
    w = torch.rand((len(p.lens), width), device="cuda") if given else None
    out = w if alias else torch.full((len(p.lens), width), 7.0, device="cuda")
    w64 = f64(w) if given else None
    want, mag = partial.key_weights(f64(p.q), f64(p.k), p.table if p.t_table is not None else None,
                                    np.minimum(p.lens, width), lse.astype(np.float64), decay, w64, f64(out), p.scale)
    kvshot.key_weights(p.desc, p.q, p.k, p.t_table, p.t_lens, torch.from_numpy(lse).cuda(), decay, width, w, out)
    check(p, code)
    terms = p.q.shape[1] * p.hq + 1
    assert np.all(np.abs(f64(out) - want) <= (2.0 ** -16 * mag + 2.0 ** -21 + terms * 2.0 ** -24) * np.abs(want) + 1e-30)
    return out


@pytest.mark.parametrize("hq,hkv", [(32, 8), (8, 8), (28, 4), (8, 1), (32, 1), (34, 2), (9, 3)])
@pytest.mark.parametrize("query", [1, 3, 12, 33])
def test_weights(hq, hkv, query):
    run_weights(Problem([0, 1, 127, 128, 129, 300], 16, hq=hq, hkv=hkv, nodes=query, query=query, seed=hq + query), 0.75)


@pytest.mark.parametrize("page", [8, 16, 64, 128, 192, 256])
@pytest.mark.parametrize("query", [2, 16])
def test_weights_pages(page, query):
    run_weights(Problem(LENS, page, nodes=query, query=query, seed=page))


@pytest.mark.parametrize("query", [1, 20, 64])
def test_weights_of_a_contiguous_cache(query):
    run_weights(Problem([777, 5, 0, 128], 16, nodes=query, query=query, contiguous=True, seed=query), 0.5)


@pytest.mark.parametrize("page", [8, 64, 192])
@pytest.mark.parametrize("query", [3, 6, 11, 16])
def test_weights_of_many_caches(page, query):
    run_weights(Problem([0, 1, 127, 128, 129, 300] * 30, page, hq=8, hkv=2, nodes=query, query=query, seed=query), 0.5)


@pytest.mark.parametrize("query", [1, 64])
def test_weights_of_a_long_cache(query):
    run_weights(Problem([3001], 64, nodes=query, query=query, seed=1, hq=8, hkv=2), 0.5)


@pytest.mark.parametrize("query", [1, 24])
def test_weights_forms(query):
    p = Problem([300, 40], 16, nodes=query, query=query, scale=0.2)
    run_weights(p, 1.0, given=False)
    run_weights(p, 1.0, alias=True)
    a, b = run_weights(p, 0.0, given=False), run_weights(p, 0.0, given=False)
    assert torch.equal(a, b)
    out = torch.empty((2, 300), device="cuda")
    nan = torch.full_like(out, float("nan"))
    kvshot.key_weights(p.desc, p.q, p.k, p.t_table, p.t_lens, torch.from_numpy(some_lse(p)).cuda(), 0.0, 300, nan, out)
    check(p)
    assert torch.equal(out[0], a[0, :300])


@pytest.mark.parametrize("query", [2, 20])
def test_weights_of_empty_rows(query):
    p = Problem([300, 40], 16, nodes=query, query=query)
    lse = some_lse(p)
    lse[:, 0] = -np.inf
    lse[0, 1, 3] = -np.inf
    run_weights(p, 1.0, lse=lse)
    lse[:] = -np.inf
    out = run_weights(p, 1.0, lse=lse, given=False)
    assert float(out[0, :300].abs().max()) == 0


def test_weights_sum_to_what_the_softmax_gives():
    p = Problem([500, 33], 16, nodes=3, query=3)
    lse = np.zeros((2, 3, 32), np.float32)
    size = kvshot.workspace_size(p.desc)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    p.desc.workspace, p.desc.workspace_bytes = ws.data_ptr(), size
    out, z = torch.empty_like(p.q), torch.empty(p.q.shape[:3], device="cuda")
    kvshot.draft_attn(p.desc, p.q, p.k, p.v, p.t_table.clamp(min=0), p.t_lens, p.dk, p.dv, None, out, z)
    check(p)
    lse = z.cpu().numpy()
    w = run_weights(p, 1.0, given=False, lse=lse)
    # what is missing of one per row and head are the weights of the draft keys
    draft = 0.0
    for n in range(3):
        for head in range(32):
            s = p.scale * (f64(p.dk)[:, head // 4, :n + 1] @ f64(p.q)[:, n, head][:, :, None])[..., 0]
            draft += np.exp(s - lse[:, n, head][:, None]).sum()
    assert abs(float(w[0, :500].sum() + w[1, :33].sum()) + draft - 2 * 3 * 32) <= 1e-3


def test_weights_records_what_it_has_no_room_for():
    p = Problem([300, 40], 16, nodes=2, query=2)
    run_weights(p, 1.0, width=100, code=kvshot.KVSHOT_ERR_DEVICE_BOUNDS)
    p.err.zero_()
    p.t_table[0, 3] = p.num_pages  # that page is passed over
    out = torch.full((2, 300), 7.0, device="cuda")
    kvshot.key_weights(p.desc, p.q, p.k, p.t_table, p.t_lens, torch.from_numpy(some_lse(p)).cuda(), 1.0, 300, None, out)
    check(p, kvshot.KVSHOT_ERR_DEVICE_BOUNDS)
    assert float(out[0, 48:64].min()) == 7.0 and float(out[0, :48].max()) < 7.0


# ------------------------------------------------------------ eviction

def some_kept(lens, counts, width, seed=0):
    rng = np.random.default_rng(seed)
    kept = np.full((len(lens), width), -1, np.int32)
    for c, (n, m) in enumerate(zip(lens, counts)):
        kept[c, :m] = np.sort(rng.permutation(int(n))[:m])
    return kept


def run_evict(p, counts, kept=None, in_place=True, weights=True, free=True, code=0, width_out=None):
    C = len(p.lens)
    width = max(1, int(max(counts)))
    kept = some_kept(p.lens, counts, width, 3) if kept is None else kept
    W = max(1, int(p.lens.max())) + 1
    w = torch.rand((C, W), device="cuda")
    rng = np.random.default_rng(1)
    if in_place:
        k_out, v_out, table_out, t_out, w_out = p.k, p.v, p.table, p.t_table, w
    else:
        used = -(-np.maximum(np.asarray(counts), 0) // p.page)
        pool = int(used.sum()) + 2
        ids = rng.permutation(pool)
        table_out = np.full((C, max(1, int(used.max()))), -3, np.int32)
        table_out[np.arange(table_out.shape[1])[None] < used[:, None]] = ids[:int(used.sum())]
        t_out = p.ints(table_out)
        k_out, v_out = (torch.full((pool, p.hkv, p.page, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        w_out = torch.full((C, width_out or width), 7.0, device="cuda")
    d = kvshot.make_evict_desc(num_caches=C, hkv=p.hkv, page_size=p.page, max_pages_per_seq=p.table.shape[1],
                               num_pages=p.num_pages, max_pages_out=table_out.shape[1], num_pages_out=k_out.shape[0],
                               max_kept=kept.shape[1], weights_len=W, weights_len_out=w_out.shape[1], err_flag=p.err)
    fl = torch.full((p.num_pages,), -9, dtype=torch.int32, device="cuda")
    fl[:len(p.free)] = p.ints(p.free)
    fc, fc_out = p.ints([len(p.free)]), p.ints([-1])
    lens_out = p.t_lens.clone() if in_place else torch.full((C,), 77, dtype=torch.int32, device="cuda")
    bits = lambda x: x.view(torch.int16).cpu().numpy()  # noqa: E731
    want = partial.cache_evict(bits(p.k), bits(p.v), p.table, p.lens, kept, counts, f64(w), bits(k_out), bits(v_out), table_out,
                               f64(w_out), fl.cpu().numpy(), len(p.free))
    kvshot.cache_evict(d, p.k, p.v, p.t_table, p.t_lens if not in_place else lens_out, p.ints(kept), p.ints(counts),
                       w if weights else None, k_out, v_out, t_out, lens_out, w_out if weights else None, fl if free else None,
                       fc if free else None, fc_out if free else None)
    check(p, code)
    got = (bits(k_out), bits(v_out), lens_out.cpu().numpy(), f64(w_out), fl.cpu().numpy(), int(fc_out.item()))
    for i, (x, y) in enumerate(zip(got, want)):
        if (i == 3 and not weights) or (i >= 4 and not free):
            continue
        assert np.array_equal(x, y), i
    return got


@pytest.mark.parametrize("page", [1, 8, 16, 24, 64, 256])
@pytest.mark.parametrize("in_place", [True, False])
def test_evict(page, in_place):
    p = Problem(LENS + [700], page, hq=3, hkv=3, seed=page)
    run_evict(p, [0, 1, 3, 8, 9, 1, 63, 40, 130, 31, 0, 512], in_place=in_place)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("weights,free", [(True, False), (False, True), (False, False)])
def test_evict_without_weights_or_free_pages(in_place, weights, free):
    run_evict(Problem([300, 20], 16), [100, 20], in_place=in_place, weights=weights, free=free)


@pytest.mark.parametrize("in_place", [True, False])
def test_evict_long_caches(in_place):
    run_evict(Problem([9000, 3001], 64, hq=2, hkv=2), [5000, 2999], in_place=in_place)
    p = Problem([5000], 16, hq=1, hkv=1)
    for kept in (np.arange(4999), np.arange(1, 5000), np.r_[0, np.arange(2, 5000)]):  # rows that move by one or not at all
        run_evict(p, [4999], kept.astype(np.int32)[None], in_place=False)
        q = Problem([5000], 16, hq=1, hkv=1)
        run_evict(q, [4999], kept.astype(np.int32)[None])


def test_evict_many_caches():
    lens = np.random.default_rng(0).integers(0, 90, size=1024)
    run_evict(Problem(lens, 8, hq=1, hkv=1), lens // 3)


def test_evict_refuses_a_count_that_does_not_fit_and_keeps_the_cache():
    p = Problem([300, 50, 100], 16)
    before = p.k.clone(), p.v.clone()
    d = kvshot.make_evict_desc(num_caches=3, hkv=8, page_size=16, max_pages_per_seq=p.table.shape[1], num_pages=p.num_pages,
                               max_kept=60, err_flag=p.err)
    kept = some_kept([300, 50, 100], [60, 50, 60], 60)
    fl, fc = torch.full((p.num_pages,), -9, dtype=torch.int32, device="cuda"), p.ints([0])
    lens = p.t_lens.clone()
    counts = p.ints([61, 51, -1])
    kvshot.cache_evict(d, p.k, p.v, p.t_table, lens, p.ints(kept), counts, None, p.k, p.v, p.t_table, lens, None, fl, fc, fc)
    check(p, kvshot.KVSHOT_ERR_DEVICE_BOUNDS)
    assert torch.equal(lens, p.t_lens) and int(fc.item()) == 0 and int(fl.max()) == -9
    for x, y in zip(before, (p.k, p.v)):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_evict_bad_lists_stay_in_the_cache():
    p = Problem([300, 50], 16)
    d = kvshot.make_evict_desc(num_caches=2, hkv=8, page_size=16, max_pages_per_seq=p.table.shape[1], num_pages=p.num_pages,
                               max_kept=60, err_flag=p.err)
    kept = some_kept([300, 50], [60, 50], 60)
    kept[0, 7], kept[0, 20], kept[0, 30] = 2 ** 31 - 1, -5, 300
    other = p.k[p.t_table[1, :4].long()].clone()
    lens = p.t_lens.clone()
    kvshot.cache_evict(d, p.k, p.v, p.t_table, lens, p.ints(kept), p.ints([60, 50]), None, p.k, p.v, p.t_table, lens, None, None,
                       None, None)
    check(p, kvshot.KVSHOT_ERR_DEVICE_BOUNDS)
    assert torch.equal(other.view(torch.int16), p.k[p.t_table[1, :4].long()].view(torch.int16))  # (all kept: nothing moves)
    assert lens.tolist() == [60, 50]


def test_evict_records_a_page_outside_the_pool_among_those_given_back():
    p = Problem([100, 40], 16)
    p.table[0, 5] = p.num_pages  # page 5 of 7; the first 30 kept tokens come from before it, and need 2
    p.t_table = p.ints(p.table)
    kept = np.stack([np.arange(30), np.arange(30)]).astype(np.int32)
    got = run_evict(p, [30, 30], kept=kept, code=kvshot.KVSHOT_ERR_DEVICE_BOUNDS)
    assert p.num_pages in got[4] and got[5] == len(p.free) + 5 + 1
