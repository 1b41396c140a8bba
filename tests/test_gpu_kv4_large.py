"""4-bit cache: the kernels that large calls take (four heads to a thread, an extension of two launches), and a window with
32 query rows.

Store and load: the bytes and values that small calls give (those are held to the oracle in tests/test_gpu_kv4.py), and the
oracle's for a sample of the tokens.  Extension: the oracle's integers.  Attention: the bounds of tests/test_gpu_kv4.py.
"""
import numpy as np
import pytest
import torch

from oracle import kv4
from paper_2604_26412_gb300 import kvshot
from tests.test_gpu_kv4 import D, Case, _i32, _random_extend, _run_extend, _tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,hkv,page,fused,exps", [
    (10007, 8, 64, 32, (0, 0)), (80001, 1, 16, 0, (-3, 2)), (40003, 2, 48, 4, (0, 0)), (26001, 3, 32, 0, (2, -1)),
    (19000, 5, 16, 0, (0, 0)), (14001, 6, 256, 3, (0, 7)), (11501, 7, 128, 0, (0, 0)),
])
def test_many_tokens_are_stored_and_loaded_as_few(t, hkv, page, fused, exps):
    """At least 80000 tokens x heads: more than fill every SM with four heads to a thread (77824 on 152 SMs)."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert t * hkv * (D // 8) // 4 >= sms * 2048  # the large kernels' calls
    gen = torch.Generator("cuda").manual_seed(t)
    rng = np.random.default_rng(t)
    pages = -(-t // page) + 3
    size = torch.exp2(torch.randint(-12, 12, (t, fused + 2 * hkv, 8), device="cuda", generator=gen).float())
    qkv = (torch.randn((t, fused + 2 * hkv, D), device="cuda", generator=gen) * size.repeat_interleave(16, -1)).to(torch.bfloat16)
    k, v = qkv[:, fused:fused + hkv], qkv[:, fused + hkv:]
    slots = rng.permutation(pages * page)[:t].astype(np.int32)
    slots[rng.integers(0, t, size=5)] = -1
    slots_d = _i32(slots)
    old = torch.randint(0, 256, (pages, hkv, page // 16, 2304), dtype=torch.uint8, device="cuda", generator=gen)
    big, small = old.clone(), old.clone()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = lambda n, **kw: kvshot.make_kv4_desc(num_tokens=n, hkv=hkv, page_size=page, num_pages=pages,  # noqa: E731
                                                k_scale_exp=exps[0], v_scale_exp=exps[1], err_flag=err, **kw)
    stride = dict(k_stride=k.stride(0), v_stride=v.stride(0))
    kvshot.kv4_store(desc(t, **stride), k, v, slots_d, big)
    step = 4000 // hkv
    parts = [slice(a, min(t, a + step)) for a in range(0, t, step)]
    for p in parts:
        kvshot.kv4_store(desc(p.stop - p.start, **stride), k[p], v[p], slots_d[p].contiguous(), small)
    assert torch.equal(big, small)
    # read back into rows longer than K and V, whose rest keeps what it held
    out = torch.full((2, t, hkv + 2, D), 5.0, dtype=torch.bfloat16, device="cuda")
    row = dict(k_stride=out.stride(1), v_stride=out.stride(1))
    kvshot.kv4_load(desc(t, **row), big, slots_d, out[0], out[1])
    few = torch.full_like(out, 5.0)
    for p in parts:
        kvshot.kv4_load(desc(p.stop - p.start, **row), big, slots_d[p].contiguous(), few[0, p], few[1, p])
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    assert torch.equal(out, few) and bool((out[:, :, hkv:] == 5.0).all())
    pick = np.arange(t)[::37]
    live = slots[pick] >= 0
    for x, e, o in ((k, exps[0], out[0]), (v, exps[1], out[1])):
        codes, scales = kv4.quantise(x[torch.from_numpy(pick).cuda()].double().cpu().numpy(), e)
        want = kv4.values(codes, scales, e) * live[:, None, None]
        assert np.array_equal(o[torch.from_numpy(pick).cuda(), :hkv].double().cpu().numpy(), want)


@pytest.mark.parametrize("bad", [-2, 2 ** 31 - 1])
def test_many_tokens_with_slots_outside_the_cache(bad):
    t, hkv, pages = 20000, 5, 1251
    k = torch.randn((t, hkv, D), device="cuda").to(torch.bfloat16)
    slots = np.arange(t, dtype=np.int32)
    slots[777] = bad
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache = torch.full((pages, hkv, 1, 2304), 0x55, dtype=torch.uint8, device="cuda")
    d = kvshot.make_kv4_desc(num_tokens=t, hkv=hkv, page_size=16, num_pages=pages, err_flag=err)
    kvshot.kv4_store(d, k, k, _i32(slots), cache)
    assert int(err.item()) == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    assert bool((cache[t // 16:] == 0x55).all())  # the slots past the stored ones
    page = kv4.unpack(cache[777 // 16:777 // 16 + 1].cpu().numpy())
    assert (page[0][0, :, 777 % 16] == 5).all() and (page[1][0, :, 777 % 16] == 0x55).all()
    err.zero_()
    out = torch.full((2, t, hkv, D), 9.0, dtype=torch.bfloat16, device="cuda")
    kvshot.kv4_load(d, cache, _i32(slots), out[0], out[1])
    assert int(err.item()) == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    assert bool((out[:, 777] == 0).all()) and not bool((out[0, :777] == 9).all())


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("c,page,max_len,max_new", [
    (1, 16, 0, 200_000), (1, 1, 70_000, 140_000), (3, 7, 100_000, 120_000), (256, 16, 0, 1500), (300, 16, 9000, 8),
    (1000, 32, 6000, 300), (1024, 64, 16_000, 5), (1024, 1, 300, 2), (257, 48, 0, 1100),
])
def test_large_extensions_match_the_oracle(c, page, max_len, max_new, in_place):
    """More than 131072 table entries or tokens, the most that one cluster takes."""
    rng = np.random.default_rng(c * 1000 + page + max_new)
    lens, new, table, free, pages = _random_extend(rng, c, page, max_len, max_new)
    if c == 1:
        new[0] = max_new - 3
        lens, new, table, free, pages = _fixed_extend(rng, lens, new, page)
    t = int(new.sum()) + int(rng.integers(0, 9))
    assert max(t, table.size) > 131072
    ref = kv4.extend(lens, new, table, free, len(free), page, t)
    err, got = _run_extend(lens, new, table, free, len(free), page, t, pages, in_place)
    assert err == 0
    want = [ref[0], ref[1], np.array([ref[2]]), *ref[3:]]
    for name, g, w in zip(("lens", "table", "count", "start", "slots", "caches", "positions"), got, want):
        assert np.array_equal(g, w), name


def _fixed_extend(rng, lens, new, page):
    used, after = -(-lens // page), -(-(lens + new) // page)
    ids = rng.permutation(int(after.sum()) + 5)
    table = np.full((len(lens), int(after.max()) + 1), -1)
    held = np.arange(table.shape[1])[None, :] < used[:, None]
    table[held] = ids[:held.sum()]
    return lens, new, table, ids[held.sum():], len(ids)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("what", ["pages", "row", "tokens", "negative count", "free id"])
def test_large_extensions_that_cannot_be_met_take_nothing(what, in_place):
    rng = np.random.default_rng(6)
    lens, new, table, free, pages = _random_extend(rng, 500, 16, 6000, 300)
    count, t = len(free), int(new.sum()) + 3
    assert table.size > 131072
    if what == "pages":
        count = int((-(-(lens + new) // 16) - -(-lens // 16)).sum()) - 1
    elif what == "row":
        new[3] = table.shape[1] * 16 + 1
        t += int(new[3])
    elif what == "tokens":
        t = int(new.sum()) - 1
    elif what == "negative count":
        new[499] = -1
    else:
        free[count // 2] = pages
    err, got = _run_extend(lens, new, table, free, count, 16, t, pages, in_place)
    assert err == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    for g, w in zip(got, [lens, table, np.array([count]), np.zeros(501), *[np.full(t, -1)] * 3]):
        assert np.array_equal(g, w)


@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 1), (16, 4), (100, 130), (128, 16), (300, 0), (1000, 7)])
@pytest.mark.parametrize("shape", ["chain", "tree"])
def test_windows_with_32_rows(window, sinks, shape):
    rng = np.random.default_rng(window + sinks)
    if shape == "chain":
        Case([0, 3, 130, 256, 451], nodes=11, query=8, window=window, sinks=sinks, page=32, seed=window).check()
    else:
        Case([2, 300, 129], nodes=24, query=8, parent=_tree(rng, 3, 24, 6), window=window, sinks=sinks, seed=window).check()
