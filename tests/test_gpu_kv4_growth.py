"""Drafting over a 4-bit cache that grows: the draft tokens' places behind the grown prefix, and growth that is refused.

Positions here come from the cache's own lengths and the nodes' depths (a node of depth d stands at L + d - 1), not from
the step.  The appended q and K have to be the oracle's bits at those positions; bounds of the attention as in
tests/test_gpu_kv4.py.
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
HKV = 2


def _inputs(levels, tree=True, layers=1, lens=(40, 0, 129), paged=True, seed=3):
    spec = wl.Spec("kv4-growth", len(lens) // layers, layers, list(lens), levels, tree, paged, page_size=16, hq=8,
                   hkv=HKV, seed=seed)
    return spec, wl.make_inputs(spec, "cuda", seed=seed, tail_fill="nan")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rows(t, seed=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    return [torch.randn((t, HKV, 128), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]


def _wide(bits):
    return wl.bits_to_bf16(bits).double().numpy()


def _check(step, inp, cache):
    """The last step against append and attention at the places behind the cache's present lengths."""
    s = inp.spec
    lens, table = cache.seq_lens.cpu().numpy(), cache.page_table.cpu().numpy()
    parent = inp.tree_parent.cpu().numpy()
    depth = np.zeros(parent.shape, np.int64)
    for i in range(parent.shape[1]):
        up = parent[:, i]
        depth[:, i] = np.where(up < 0, 0, depth[np.arange(len(up)), up]) + 1
    dk = np.full((s.num_caches, s.hkv, inp.n_max, 128), 0x7FC0, np.uint16)
    dv = dk.copy()
    d = oracle.make_desc(num_caches=s.num_caches, num_seqs=s.num_seqs, hq=s.hq, hkv=s.hkv, head_dim=128, n_nodes=0,
                         n_query=0, n_max=inp.n_max, tree=s.tree, l_cap=1)
    n0 = 0
    for i, n in enumerate(step.levels):
        pos = lens[:, None] + depth[np.arange(s.num_caches) // s.layers, n0:n0 + n] - 1
        q = oracle.append(d, wl.bf16_bits(step.q_in[i]), wl.bf16_bits(step.k_in[i]), wl.bf16_bits(step.v_in[i]),
                          pos.astype(np.int32), n0, n, s.rope_base, dk, dv)
        n0 += n
        assert np.array_equal(wl.bf16_bits(step.q_rot[i]), q), i
        assert np.array_equal(wl.bf16_bits(step.draft_k[:, :, n0 - n:n0]), dk[:, :, n0 - n:n0]), i
        for c in range(s.num_caches):
            slots = [table[c, j // cache.page_size] * cache.page_size + j % cache.page_size for j in range(lens[c])]
            k, v = (x.double().cpu().numpy().swapaxes(0, 1) for x in cache.values(_i32(slots)))
            par = parent[c // s.layers, :n0] if s.tree else None
            out, lse = kv4.attn(_wide(q[c]), k, v, _wide(dk[c, :, :n0]), _wide(dv[c, :, :n0]), par, step.window,
                                step.sinks, 128 ** -0.5)
            o, l = step.out[i][c].double().cpu().numpy(), step.lse[i][c].double().cpu().numpy()
            assert np.abs(o - out).max() <= OUT_MAX_ABS, (i, c)
            assert np.linalg.norm(o - out) <= OUT_REL_L2 * np.linalg.norm(out), (i, c)
            assert np.abs(l - lse).max() <= LSE_MAX_ABS, (i, c)
    assert step.error_code() == 0 and cache.error_code() == 0


# ------------------------------------------------------------------ places of the draft tokens

@pytest.mark.parametrize("mode", ["per_depth", "whole"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 5)])
@pytest.mark.parametrize("levels,tree,layers", [([2, 3], True, 1), ([1, 1, 1], False, 3), ([2, 2, 4, 4, 1], True, 1)])
def test_draft_tokens_stand_behind_the_grown_prefix(mode, window, sinks, levels, tree, layers):
    _, inp = _inputs(levels, tree, layers)
    cache = user.of_inputs(inp, spare_pages=8, spare_tokens=60)
    step = DraftStep(inp, mode=mode, target_kv4=cache, window=window, sinks=sinks)
    step.run()
    _check(step, inp, cache)
    for new in ([3, 1, 0], [0, 17, 8]):
        cache.grow(_i32(new), *_rows(sum(new), seed=sum(new)))
        step.run()
        _check(step, inp, cache)


def test_draft_tokens_stand_behind_the_grown_prefix_in_a_replayed_graph():
    _, inp = _inputs([2, 3])
    cache = user.of_inputs(inp, spare_pages=8, spare_tokens=40)
    step = DraftStep(inp, target_kv4=cache, window=30, sinks=2)
    new, (k, v) = _i32([2, 5, 1]), _rows(8)
    cache.grow(new, k, v)  # (uncaptured: what a first call sets up)
    step.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.grow(new, k, v)
        step.run()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        _check(step, inp, cache)


def test_a_cache_of_other_lengths_than_the_inputs():
    _, inp = _inputs([2, 3])
    cache = user.Kv4Cache(3, HKV, 20, 8, max_tokens=100)
    cache.grow(_i32([7, 70, 20]), *_rows(97))
    step = DraftStep(inp, target_kv4=cache)
    step.run()
    _check(step, inp, cache)


@pytest.mark.parametrize("handle", [False, True])
def test_a_step_on_another_stream(handle):
    """The places are found on the step's stream, after the growth that stands there before it."""
    _, inp = _inputs([2, 3])
    cache = user.of_inputs(inp, spare_pages=8, spare_tokens=40)
    step = DraftStep(inp, target_kv4=cache)
    new, (k, v) = _i32([2, 5, 1]), _rows(8)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
    on = s.cuda_stream if handle else s
    cache.grow(new, k, v, stream=on)
    step.run(on)
    torch.cuda.synchronize()
    _check(step, inp, cache)


def test_the_steps_of_the_other_caches_keep_their_places():
    _, inp = _inputs([2, 3])
    step = DraftStep(inp)
    assert all(a is b for a, b in zip(step.pos, inp.positions))


# ------------------------------------------------------------------ growth that is refused

def _state(cache):
    return [x.clone() for x in (cache.seq_lens, cache.page_table, cache.free_count, cache.data)]


def _unmoved(cache, before):
    return all(torch.equal(a, b) for a, b in zip(before, _state(cache)))


def _wrong_rows(what):
    k = torch.zeros((4, HKV, 128), dtype=torch.bfloat16, device="cuda")
    flat = torch.zeros(4 * HKV * 128 + 64, dtype=torch.bfloat16, device="cuda")
    return {
        "type": k.float(), "heads": k[:, :1], "order": k.transpose(1, 2), "host": k.cpu(),
        "many": torch.zeros((200, HKV, 128), dtype=torch.bfloat16, device="cuda"),
        "shared": k[:1].expand(4, HKV, 128),
        "address": flat[4:4 + 4 * HKV * 128].view(4, HKV, 128),
        "stride": torch.as_strided(flat, (4, HKV, 128), (HKV * 128 + 4, 128, 1)),
        "overlap": torch.as_strided(flat, (4, HKV, 128), (128, 128, 1)),
        "dims": k[0],
    }[what]


@pytest.mark.parametrize("what", ["type", "heads", "order", "host", "many", "shared", "address", "stride", "overlap", "dims"])
@pytest.mark.parametrize("which", ["k", "v"])
def test_growth_with_wrong_rows_moves_nothing(what, which):
    cache = user.Kv4Cache(3, HKV, 20, 8, max_tokens=100)
    before = _state(cache)
    bad = _wrong_rows(what)
    good = torch.zeros((bad.shape[0], HKV, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises((ValueError, kvshot.KvshotError)):
        cache.grow(_i32([3, 1, 0]), *((bad, good) if which == "k" else (good, bad)))
    assert _unmoved(cache, before)


def test_growth_with_fewer_rows_than_tokens_moves_nothing():
    cache = user.Kv4Cache(3, HKV, 20, 8, max_tokens=100)
    cache.grow(_i32([20, 3, 40]), *_rows(63))
    before = _state(cache)
    cache.grow(_i32([3, 1, 0]), *_rows(3))
    assert _unmoved(cache, before)
    assert cache.error_code() == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    assert all(bool((m == -1).all()) for m in (cache.slots, cache.token_cache, cache.positions))
    assert int(cache.token_start.abs().max()) == 0


def test_maps_past_the_new_tokens_say_so():
    cache = user.Kv4Cache(3, HKV, 20, 8, max_tokens=100)
    cache.grow(_i32([20, 3, 40]), *_rows(63))
    cache.grow(_i32([3, 0, 2]), *_rows(7))
    assert cache.positions.tolist() == [20, 21, 22, 40, 41] + [-1] * 95
    assert cache.token_cache.tolist() == [0, 0, 0, 2, 2] + [-1] * 95
    assert cache.slots[5:].tolist() == [-1] * 95 and int(cache.slots[:5].min()) >= 0
    assert cache.error_code() == 0


@pytest.mark.parametrize("sizes", [dict(k_scale_exp=65), dict(v_scale_exp=-65), dict(hkv=16385, num_pages=1),
                                   dict(max_tokens=-1), dict(num_caches=0), dict(max_pages_per_seq=0),
                                   dict(num_caches=1025)])
def test_sizes_that_no_call_takes_are_refused_at_once(sizes):
    with pytest.raises((ValueError, kvshot.KvshotError)):
        user.Kv4Cache(**(dict(num_caches=3, hkv=HKV, num_pages=20, max_pages_per_seq=8, max_tokens=100) | sizes))


def _wrong_counts(what):
    return {
        "int64": torch.tensor([3, 1, 0], device="cuda"), "host": torch.tensor([3, 1, 0], dtype=torch.int32),
        "short": _i32([3]), "long": _i32([3, 1, 0, 0]), "strided": _i32([3, 9, 1, 9, 0, 9])[::2],
        "float": torch.tensor([3.0, 1.0, 0.0], device="cuda"), "dims": _i32([[3, 1, 0]]),
    }[what]


@pytest.mark.parametrize("what", ["int64", "host", "short", "long", "strided", "float", "dims"])
def test_counts_of_another_type_or_shape_are_refused(what):
    cache = user.Kv4Cache(3, HKV, 20, 8, max_tokens=100)
    before = _state(cache)
    for call in (lambda n: cache.grow(n, *_rows(4)), cache.extend):
        with pytest.raises(ValueError):
            call(_wrong_counts(what))
    assert _unmoved(cache, before)


@pytest.mark.parametrize("what", ["int64", "host", "strided", "float", "dims"])
def test_slots_of_another_type_or_shape_are_refused(what):
    cache = user.Kv4Cache(3, HKV, 20, 8, max_tokens=100)
    before = _state(cache)
    with pytest.raises(ValueError):
        cache.values(_wrong_counts(what))
    with pytest.raises(ValueError):
        cache.store(*_rows(1), slots=_wrong_counts(what))
    assert _unmoved(cache, before)


def test_an_error_is_reported_once():
    cache = user.Kv4Cache(3, HKV, 20, 8, max_tokens=100)
    cache.grow(_i32([100, 100, 100]), *_rows(100))
    assert cache.error_code() == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    cache.grow(_i32([3, 1, 0]), *_rows(4))
    assert cache.error_code() == 0 and cache.seq_lens.tolist() == [3, 1, 0]


@pytest.mark.parametrize("handle", [False, True])
def test_values_on_another_stream_are_written_by_it_alone(handle):
    """Memory that the current stream has let go of, with work on it still to come, is not another stream's to write."""
    cache = user.Kv4Cache(3, HKV, 600, 200, max_tokens=4096)
    cache.grow(_i32([3000, 1000, 96]), *_rows(4096))
    want = cache.values(cache.slots)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    old = [torch.empty((4096, HKV, 128), dtype=torch.bfloat16, device="cuda") for _ in range(8)]
    torch.cuda._sleep(200_000_000)
    for x in old:
        x.fill_(7.0)
    del x, old
    got = cache.values(cache.slots, stream=s.cuda_stream if handle else s)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
