"""GPU parity of the 4-bit cache's entry points with the fp64 oracle (oracle/kv4.py).

Tolerances.  Integers, and the values of the cache (exact in bf16), have to be equal.  Attention: as for a bf16 cache
(tests/gpu_helpers.py): out max-abs 2e-2 and rel-L2 5e-3, lse 1e-3.  The cache's values are exact in f16 and so is q
here (|q| >= 2^-14 or 0 after rounding to f16 loses 2^-25 at most); P rounded to f16 is off by 2^-12 of itself, out by
2^-12 of the values' size and by its own rounding to bf16, 2^-9: rel-L2 below 2e-3, half of what is allowed.
"""
import numpy as np
import pytest
import torch

from oracle import kv4
from paper_2604_26412_gb300 import kvshot
from tests.gpu_helpers import LSE_MAX_ABS, OUT_MAX_ABS, OUT_REL_L2

pytestmark = pytest.mark.gpu
D = 128


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


# ------------------------------------------------------------------ extend

def _run_extend(lens, new, table, free, count, page, max_tokens, num_pages, in_place=False, maps=True):
    c, per = table.shape
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    d = kvshot.make_extend_desc(num_caches=c, page_size=page, max_pages_per_seq=per, num_pages=num_pages,
                                max_tokens=max_tokens, num_free=len(free), err_flag=err)
    a = [_i32(lens), _i32(new), _i32(table), _i32(free if len(free) else [0]), _i32([count])]
    outs = [a[0], a[2], a[4]] if in_place else [torch.full_like(x, -77) for x in (a[0], a[2], a[4])]
    start = torch.full((c + 1,), -77, dtype=torch.int32, device="cuda")
    m = [torch.full((max_tokens,), -77, dtype=torch.int32, device="cuda") for _ in range(3)]
    kvshot.cache_extend(d, *a, *outs, start, *(m if maps else [None] * 3))
    torch.cuda.synchronize()
    host = lambda x: x.cpu().numpy()  # noqa: E731
    return int(err.item()), [host(x) for x in (*outs, start, *m)]


def _random_extend(rng, c, page, max_len, max_new):
    lens, new = rng.integers(0, max_len, size=c, endpoint=True), rng.integers(0, max_new, size=c, endpoint=True)
    used, after = -(-lens // page), -(-(lens + new) // page)
    per = max(1, int(after.max()) + rng.integers(0, 2))
    need = int((after - used).sum())
    ids = rng.permutation(int(used.sum()) + need + 5)
    table = np.full((c, per), -1)
    held = np.arange(per)[None, :] < used[:, None]
    table[held] = ids[:held.sum()]
    free = ids[held.sum():]
    return lens, new, table, free, len(ids)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("c,page,max_len,max_new", [
    (1, 16, 0, 0), (1, 16, 0, 1), (1, 16, 100, 40), (3, 1, 9, 9), (5, 7, 60, 33), (31, 16, 100, 3), (33, 64, 700, 8),
    (64, 16, 900, 8), (257, 16, 0, 100), (1000, 32, 200, 5), (1024, 128, 300, 2), (2, 16, 0, 40000),
])
def test_extend_matches_oracle(c, page, max_len, max_new, in_place):
    rng = np.random.default_rng(c * 1000 + page + max_new)
    lens, new, table, free, pages = _random_extend(rng, c, page, max_len, max_new)
    t = int(new.sum()) + int(rng.integers(0, 9))
    ref = kv4.extend(lens, new, table, free, len(free), page, t)
    err, got = _run_extend(lens, new, table, free, len(free), page, t, pages, in_place)
    assert err == 0
    want = [ref[0], ref[1], np.array([ref[2]]), *ref[3:]]
    for name, g, w in zip(("lens", "table", "count", "start", "slots", "caches", "positions"), got, want):
        assert np.array_equal(g, w), name


def test_extend_without_maps():
    rng = np.random.default_rng(5)
    lens, new, table, free, pages = _random_extend(rng, 9, 16, 100, 20)
    err, got = _run_extend(lens, new, table, free, len(free), 16, 500, pages, maps=False)
    ref = kv4.extend(lens, new, table, free, len(free), 16, 500)
    assert err == 0 and np.array_equal(got[1], ref[1]) and np.array_equal(got[3], ref[3])


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("what", ["pages", "row", "tokens", "negative length", "negative count", "free id", "count",
                                  "last page id"])
def test_extend_that_cannot_be_met_takes_nothing(what, in_place):
    rng = np.random.default_rng(6)
    lens, new, table, free, pages = _random_extend(rng, 40, 16, 100, 30)
    lens[7], new[7] = 5, 3  # joins a page
    table[7, 0] = 1
    count, t = len(free), int(new.sum()) + 3
    if what == "pages":
        count = int((-(-(lens + new) // 16) - -(-lens // 16)).sum()) - 1
    elif what == "row":
        new[3] = table.shape[1] * 16 + 1
        t += int(new[3])
    elif what == "tokens":
        t = int(new.sum()) - 1
    elif what == "negative length":
        lens[39] = -2
    elif what == "negative count":
        new[0] = -1
    elif what == "free id":
        free[count - 2] = pages
    elif what == "count":
        count = len(free) + 1
    else:
        table[7, 0] = -1
    err, got = _run_extend(lens, new, table, free, count, 16, t, pages, in_place)
    assert err == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    for g, w in zip(got, [lens, table, np.array([count]), np.zeros(41), *[np.full(t, -1)] * 3]):
        assert np.array_equal(g, w)


# ------------------------------------------------------------------ store, load

def _special_rows(rng, t, hkv):
    """Ordinary rows of several sizes, with ties, zeros, tiny, huge and subnormal numbers among them."""
    x = rng.normal(size=(t, hkv, D)) * np.exp2(rng.integers(-12, 12, size=(t, hkv, 8)).repeat(16, -1))
    x.reshape(-1, 16)[::7] = 0
    x.reshape(-1, 16)[3::11] = rng.choice([6, 0.25, -0.75, 1.25, 1.75, -2.5, 3.5, 5, 4.5], size=16)
    x.reshape(-1, 16)[5::13, 2] *= 2.0 ** 100
    x.reshape(-1, 16)[6::17] *= 2.0 ** -130
    return torch.from_numpy(x).to(torch.bfloat16)


@pytest.mark.parametrize("t,hkv,page,pages,fused,exps", [
    (1, 1, 16, 1, 0, (0, 0)), (5, 2, 16, 3, 0, (0, 0)), (33, 8, 32, 4, 0, (-3, 2)), (100, 3, 64, 3, 5, (0, -1)),
    (1000, 4, 256, 5, 0, (7, -9)), (77, 8, 48, 3, 32, (0, 0)), (64, 1, 16, 9, 2, (64, -64)),
])
def test_store_and_load(t, hkv, page, pages, fused, exps):
    rng = np.random.default_rng(t + page)
    heads = fused + 2 * hkv
    qkv = _special_rows(rng, t, heads).cuda()
    k, v = qkv[:, fused:fused + hkv], qkv[:, fused + hkv:]
    slots = rng.permutation(pages * page)[:t].astype(np.int32)
    if t > 4:
        slots[3] = -1
    cache0 = torch.from_numpy(rng.integers(0, 256, size=(pages, hkv, page // 16, 2304), dtype=np.uint8)).cuda()
    cache = cache0.clone()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    sizes = dict(num_tokens=t, hkv=hkv, page_size=page, num_pages=pages, k_scale_exp=exps[0], v_scale_exp=exps[1],
                 err_flag=err)
    kvshot.kv4_store(kvshot.make_kv4_desc(**sizes, k_stride=k.stride(0), v_stride=v.stride(0)), k, v, _i32(slots), cache)
    out = torch.full((2, t, hkv + 2, D), 5.0, dtype=torch.bfloat16, device="cuda")  # rows longer than K, V
    kvshot.kv4_load(kvshot.make_kv4_desc(**sizes, k_stride=out.stride(1), v_stride=out.stride(1)), cache, _i32(slots),
                    out[0], out[1])
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    # the cache: the stored slots hold the oracle's codes, the others what they held
    want = [x.copy() for x in kv4.unpack(cache0.cpu().numpy())]
    at = slots >= 0
    pg, off = slots[at] // page, slots[at] % page
    for x, e, i in ((k, exps[0], 0), (v, exps[1], 2)):
        codes, scales = kv4.quantise(x.double().cpu().numpy()[at], e)
        want[i][pg, :, off], want[i + 1][pg, :, off] = codes, scales
    got = kv4.unpack(cache.cpu().numpy())
    for name, g, w in zip(("k codes", "k scales", "v codes", "v scales"), got, want):
        assert np.array_equal(g, w), name
    # and read back
    for i, e in ((0, exps[0]), (1, exps[1])):
        ref = np.zeros((t, hkv, D))
        ref[at] = kv4.values(want[2 * i][pg, :, off], want[2 * i + 1][pg, :, off], e)
        y = out[i, :, :hkv].double().cpu().numpy()
        assert np.array_equal(y, ref)
        assert (out[i, :, hkv:] == 5.0).all()


def test_store_of_infinities_and_nan():
    k = torch.zeros(2, 1, D, dtype=torch.bfloat16)
    k[0, 0, 0], k[0, 0, 16], k[0, 0, 33], k[1, 0, 5] = float("inf"), float("nan"), float("-inf"), -float("nan")
    k[0, 0, 1], k[0, 0, 17], k[1, 0, 100] = 300.0, 1.0, 3.0e38
    v = -k
    cache = torch.zeros((1, 1, 1, 2304), dtype=torch.uint8, device="cuda")
    d = kvshot.make_kv4_desc(num_tokens=2, hkv=1, page_size=16, num_pages=1)
    kvshot.kv4_store(d, k.cuda(), v.cuda(), _i32([9, 2]), cache)
    got = kv4.unpack(cache.cpu().numpy())
    for x, i in ((k, 0), (v, 2)):
        codes, scales = kv4.quantise(x.double().numpy()[:, 0], 0)
        for row, slot in ((0, 9), (1, 2)):
            assert np.array_equal(got[i + 1][0, 0, slot], scales[row])
            assert np.array_equal(got[i][0, 0, slot], codes[row])
    out = torch.empty((2, 2, 1, D), dtype=torch.bfloat16, device="cuda")
    kvshot.kv4_load(d, cache, _i32([9, 2]), out[0], out[1])
    o = out[0].float().cpu()
    assert o[0, 0, 0] == 6 * 448 and o[0, 0, 33] == -6 * 448 and torch.isnan(o[0, 0, 16:32]).all()
    assert o[1, 0, 100] == 6 * 448 and torch.isnan(o[1, 0, :16]).all() and not torch.isnan(o[1, 0, 16:]).any()


@pytest.mark.parametrize("bad", [-2, 64, 2 ** 31 - 1, -2 ** 31])
def test_slots_outside_the_cache_are_passed_over(bad):
    k = torch.randn(3, 2, D, device="cuda").to(torch.bfloat16)
    cache = torch.full((4, 2, 1, 2304), 0x55, dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    d = kvshot.make_kv4_desc(num_tokens=3, hkv=2, page_size=16, num_pages=4, err_flag=err)
    kvshot.kv4_store(d, k, k, _i32([5, bad, 40]), cache)
    torch.cuda.synchronize()
    assert int(err.item()) == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    fresh = kv4.unpack(cache.cpu().numpy())[0].reshape(4, 2, 16, D)
    touched = (fresh != 5).any(-1).any(1)
    assert set(zip(*np.nonzero(touched))) == {(0, 5), (2, 8)}
    err.zero_()
    out = torch.full((2, 3, 2, D), 9.0, dtype=torch.bfloat16, device="cuda")
    kvshot.kv4_load(d, cache, _i32([5, bad, 40]), out[0], out[1])
    torch.cuda.synchronize()
    assert int(err.item()) == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    assert (out[:, 1] == 0).all() and (out[:, 0] != 9).all()


def test_slots_beyond_32_bit_offsets():
    """A cache of more than 4 GB: slots at its end."""
    pages, hkv, page = 2_100_000, 1, 16
    cache = torch.zeros(kvshot.kv4_cache_bytes(pages, hkv, page), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 2 ** 32
    k, v = (torch.randn(3, hkv, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    slots = [pages * page - 1, pages * page - 40, 7]
    d = kvshot.make_kv4_desc(num_tokens=3, hkv=hkv, page_size=page, num_pages=pages)
    kvshot.kv4_store(d, k, v, _i32(slots), cache)
    out = torch.empty((2, 3, hkv, D), dtype=torch.bfloat16, device="cuda")
    kvshot.kv4_load(d, cache, _i32(slots), out[0], out[1])
    for x, o in ((k, out[0]), (v, out[1])):
        codes, scales = kv4.quantise(x.double().cpu().numpy(), 0)
        assert np.array_equal(o.double().cpu().numpy(), kv4.values(codes, scales, 0))
    tail = cache[-2304:].cpu().numpy().reshape(1, 1, 1, 2304)
    assert np.array_equal(kv4.unpack(tail)[0][0, 0, 15], kv4.quantise(k[0].double().cpu().numpy(), 0)[0][0])


# ------------------------------------------------------------------ attention

class Case:
    """A 4-bit cache with lens[c] tokens each, garbage (NaN scales among it) in every other place."""

    def __init__(self, lens, *, seqs=None, hq=8, hkv=2, page=16, nodes=4, query=4, parent=None, window=0, sinks=0,
                 exps=(0, 0), scale=0.0, flags=0, num_ctas=0, q_std=1.0, seed=0, extra_slots=3):
        rng = np.random.default_rng(seed)
        c = len(lens)
        self.lens, self.seqs, self.hq, self.hkv, self.n, self.nq = lens, seqs or c, hq, hkv, nodes, query
        self.parent, self.window, self.sinks, self.scale = parent, window, sinks, scale
        bf = lambda *s: torch.from_numpy(rng.normal(size=s)).to(torch.bfloat16)  # noqa: E731
        per = max(1, -(-max(lens) // (page or 16)))
        self.page = page or per * 16
        used = [-(-n // page) if page else 1 for n in lens]
        total = sum(used) + 2 if page else c
        ids = rng.permutation(total)
        table = np.full((c, per), -9 if page else 0)  # entries past a cache's pages are never read
        n = 0
        for i, u in enumerate(used):
            table[i, :u] = ids[n:n + u] if page else i
            n += u
        garbage = rng.integers(0, 16, size=(4, total, hkv, self.page, D)).astype(np.uint8)
        kc, vc = garbage[0], garbage[1]
        ks, vs = (np.full((total, hkv, self.page, 8), 0x7F, np.uint8) for _ in range(2))
        self.k, self.v = [], []
        for i, length in enumerate(lens):
            x, y = bf(hkv, length, D).double().numpy(), bf(hkv, length, D).double().numpy()
            x *= 2.0 ** exps[0]
            y *= 2.0 ** exps[1]
            (xc, xs), (yc, ys) = kv4.quantise(x, exps[0]), kv4.quantise(y, exps[1])
            self.k.append(kv4.values(xc, xs, exps[0]))
            self.v.append(kv4.values(yc, ys, exps[1]))
            for j in range(length):
                at = (table[i, j // self.page] if page else i, slice(None), j % self.page)
                kc[at], ks[at], vc[at], vs[at] = xc[:, j], xs[:, j], yc[:, j], ys[:, j]
        self.cache = torch.from_numpy(kv4.pack(kc, ks, vc, vs)).cuda()
        self.table = _i32(table) if page else None
        self.q = (bf(c, query, hq, D) * q_std).to(torch.bfloat16).cuda()
        slots = nodes + extra_slots
        self.dk, self.dv = (torch.full((c, hkv, slots, D), float("nan"), dtype=torch.bfloat16) for _ in range(2))
        self.dk[:, :, :nodes], self.dv[:, :, :nodes] = bf(c, hkv, nodes, D), bf(c, hkv, nodes, D)
        self.dk, self.dv = self.dk.cuda(), self.dv.cuda()
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.desc = kvshot.make_desc(
            num_caches=c, num_seqs=self.seqs, hq=hq, hkv=hkv, n_nodes=nodes, n_query=query, n_max=slots,
            max_seq_len=max(lens), page_size=page, max_pages_per_seq=per if page else 0, num_pages=total if page else 0,
            l_cap=0 if page else self.page, scale=scale, tree=parent is not None, flags=flags, num_ctas=num_ctas,
            err_flag=self.err, k_scale_exp=exps[0], v_scale_exp=exps[1])
        size = kvshot.draft_attn_kv4_workspace_size(self.desc, window, sinks)
        assert size > 0
        self.ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN wherever it is read unwritten
        self.desc.workspace, self.desc.workspace_bytes = self.ws.data_ptr(), size
        self.out = torch.full_like(self.q, float("nan"))
        self.lse = torch.full((c, query, hq), float("nan"), device="cuda")
        self.par = _i32(parent) if parent is not None else None

    def run(self, stream=None):
        kvshot.draft_attn_kv4(self.desc, self.q, self.cache, self.table, _i32(self.lens), self.dk, self.dv, self.par,
                              self.window, self.sinks, self.out, self.lse, stream)
        torch.cuda.synchronize()
        return self.out.clone(), self.lse.clone()

    def check(self, caches=None):
        self.run()
        assert int(self.err.item()) == 0
        for c in caches if caches is not None else range(len(self.lens)):
            par = self.parent[c // (len(self.lens) // self.seqs)] if self.parent is not None else None
            out, lse = kv4.attn(self.q[c].double().cpu().numpy(), self.k[c], self.v[c],
                                self.dk[c, :, :self.n].double().cpu().numpy(),
                                self.dv[c, :, :self.n].double().cpu().numpy(), par, self.window, self.sinks,
                                self.scale or D ** -0.5)
            o, l = self.out[c].double().cpu().numpy(), self.lse[c].double().cpu().numpy()
            size = max(1.0, np.abs(self.v[c]).max() / 4 if self.v[c].size else 1.0)  # value scales other than 1
            assert np.isfinite(o).all() and np.isfinite(l).all()
            assert np.abs(o - out).max() <= OUT_MAX_ABS * size, (c, np.abs(o - out).max())
            assert np.linalg.norm(o - out) <= OUT_REL_L2 * np.linalg.norm(out), c
            assert np.abs(l - lse).max() <= LSE_MAX_ABS, (c, np.abs(l - lse).max())


def _tree(rng, seqs, n, width):
    i = np.arange(n)
    return np.where(i < width, -1, (i // width - 1) * width + rng.integers(0, width, size=(seqs, n)))


@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 127, 128, 129, 255, 257, 700])
@pytest.mark.parametrize("page", [0, 16, 64])
def test_attn_lengths(length, page):
    Case([length], page=page, nodes=3, query=1, seed=length).check()


@pytest.mark.parametrize("hq,hkv,nodes,query", [
    (1, 1, 1, 1), (2, 1, 1, 1), (8, 2, 2, 2), (8, 2, 5, 3), (8, 2, 4, 4), (28, 4, 3, 1), (16, 2, 2, 2), (8, 2, 9, 8),
    (8, 1, 6, 6), (8, 2, 13, 13), (8, 2, 24, 16), (10, 2, 16, 13), (8, 2, 17, 17), (8, 2, 24, 24), (8, 2, 31, 31),
    (8, 2, 33, 32), (8, 2, 64, 33), (8, 2, 64, 64), (16, 1, 20, 9), (64, 1, 3, 3), (48, 1, 11, 11), (200, 1, 2, 2),
])
def test_attn_row_counts(hq, hkv, nodes, query):
    """1 to 528 query rows per KV head, chains."""
    Case([150, 61], hq=hq, hkv=hkv, nodes=nodes, query=query, seed=nodes).check()


@pytest.mark.parametrize("page", [0, 16, 32, 48, 64, 128, 256])
def test_attn_page_sizes(page):
    Case([333, 0, 128, 517], page=page, nodes=7, query=3, parent=_tree(np.random.default_rng(page), 4, 7, 3),
         seed=page + 1).check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (2, 1), (5, 0), (16, 4), (100, 0), (100, 130), (128, 16),
                                          (300, 0), (1000, 7), (130, 500)])
@pytest.mark.parametrize("shape", ["chain", "tree", "whole"])
def test_attn_windows(window, sinks, shape):
    rng = np.random.default_rng(window + sinks)
    if shape == "chain":
        Case([0, 3, 130, 256, 451], nodes=9, query=2, window=window, sinks=sinks, page=32, seed=window).check()
    elif shape == "tree":
        Case([2, 300, 129], nodes=24, query=12, parent=_tree(rng, 3, 24, 6), window=window, sinks=sinks,
             seed=window).check()
    else:
        Case([260], nodes=64, query=64, parent=_tree(rng, 1, 64, 12), window=window, sinks=sinks, seed=window).check()


def test_attn_long_chain_of_drafts_in_a_window():
    for window, sinks in ((0, 0), (40, 0), (200, 20), (3, 70)):
        Case([50, 0], nodes=150, query=5, window=window, sinks=sinks, seed=9).check()


def test_attn_layers_share_a_tree():
    rng = np.random.default_rng(8)
    Case([70, 200, 133, 5, 64, 300], seqs=2, nodes=10, query=4, parent=_tree(rng, 2, 10, 4), seed=8).check()


@pytest.mark.parametrize("exps", [(0, -6), (3, 9), (-20, 30), (-64, -64), (6, 64), (0, 14)])
@pytest.mark.parametrize("nodes", [1, 12])
def test_attn_scales(exps, nodes):
    """Keys of size 2^k: scores within the range by the softmax scale."""
    Case([200, 90], nodes=nodes, query=nodes, exps=exps, scale=D ** -0.5 * 2.0 ** -max(0, exps[0]), seed=3).check()


@pytest.mark.parametrize("q_std,scale", [(30.0, 0.0), (1.0, 1.0), (300.0, 0.01), (1e-3, 0.0)])
def test_attn_sharp_and_flat(q_std, scale):
    """Running maxima that move by hundreds from tile to tile, and that do not move."""
    Case([600, 450], nodes=3, query=3, q_std=q_std, scale=scale, seed=4).check()


def test_attn_many_caches():
    rng = np.random.default_rng(11)
    lens = rng.integers(0, 90, size=300).tolist()
    Case(lens, hq=2, hkv=1, nodes=2, query=1, seed=11).check(range(0, 300, 17))


@pytest.mark.parametrize("num_ctas", [1, 2, 7, 150])
@pytest.mark.parametrize("query", [1, 12, 40])
def test_attn_grids(num_ctas, query):
    """However the work is cut, a row's result is the same row's."""
    rng = np.random.default_rng(12)
    Case([700, 33, 400], nodes=40, query=query, parent=_tree(rng, 3, 40, 12), num_ctas=num_ctas, seed=12).check()
    Case([1500], nodes=4, query=1, num_ctas=num_ctas, window=600, sinks=20, seed=13).check()


def test_attn_is_deterministic():
    c = Case([900, 350, 20], nodes=8, query=5, seed=14)
    a, b = c.run()
    for _ in range(3):
        x, y = c.run()
        assert torch.equal(a, x) and torch.equal(b, y)


def test_attn_on_another_stream():
    c = Case([400], nodes=4, query=4, seed=15)
    want = c.run()
    s = torch.cuda.Stream()
    c.out.fill_(float("nan"))
    torch.cuda.synchronize()
    kvshot.draft_attn_kv4(c.desc, c.q, c.cache, c.table, _i32(c.lens), c.dk, c.dv, c.par, 0, 0, c.out, c.lse, s)
    s.synchronize()
    assert torch.equal(want[0], c.out)


def test_attn_device_errors_are_recorded():
    c = Case([100, 40], nodes=4, query=2, seed=16)
    c.table[0, 3] = 10_000
    c.run()
    assert int(c.err.item()) == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    c = Case([100, 40], nodes=4, query=2, seed=16)
    c.lens = [101, 40]
    c.run()
    assert int(c.err.item()) == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    c = Case([100, 40], nodes=4, query=2, parent=np.array([[-1, 0, 2, 0]] * 2), seed=16)
    c.run()
    assert int(c.err.item()) == kvshot.KVSHOT_ERR_TREE


def test_attn_workspace_is_checked():
    c = Case([1000], nodes=4, query=4, seed=17)
    for ptr, size in ((None, c.ws.numel()), (c.ws.data_ptr() + 16, c.ws.numel()), (c.ws.data_ptr(), c.ws.numel() - 1)):
        c.desc.workspace, c.desc.workspace_bytes = ptr, size
        st = kvshot.draft_attn_kv4_status(c.desc, c.q, c.cache, c.table, _i32(c.lens), c.dk, c.dv, c.par, 0, 0, c.out, c.lse)
        assert st == kvshot.KVSHOT_ERR_WORKSPACE
