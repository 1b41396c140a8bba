"""Pins of the 4-bit cache's oracle (no GPU): the number formats, the quantiser, the layout, the window's mask."""
import numpy as np
import pytest
import torch

from oracle import kv4


def test_e2m1_values_are_the_formats():
    assert kv4.e2m1_value(np.arange(8)).tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert kv4.e2m1_value(np.arange(8, 16)).tolist() == [0, -0.5, -1, -1.5, -2, -3, -4, -6]
    assert kv4.E2M1.tolist() == kv4.e2m1_value(np.arange(8)).tolist()
    assert (np.diff(kv4.E4M3) > 0).all() and kv4.E4M3[1] == 2.0 ** -9 and kv4.E4M3[-1] == 448


@pytest.mark.parametrize("exp", [-64, -3, 0, 5, 64])
def test_values_are_exact_in_bf16(exp):
    codes = np.tile(np.arange(16, dtype=np.uint8), 8)
    for scale in range(1, 0x7F):
        v = kv4.values(codes, np.full(8, scale, np.uint8), exp)
        assert np.array_equal(torch.from_numpy(v).to(torch.bfloat16).double().numpy(), v)
        if exp == 0:  # and in f16
            assert np.array_equal(v.astype(np.float16).astype(np.float64), v)


def test_quantiser_is_the_nearest_by_search():
    """Scale and codes against the smallest distance over all numbers of the formats."""
    rng = np.random.default_rng(0)
    x = rng.normal(size=(64, 128)) * np.exp(rng.normal(size=(64, 1)) * 4)
    codes, scales = kv4.quantise(x, 0)
    for r in range(64):
        for b in range(8):
            blk = x[r, 16 * b:16 * b + 16]
            want = np.clip(np.abs(blk).max() / 6, 2.0 ** -9, 448)
            s = kv4.E4M3[scales[r, b]]
            assert abs(s - want) <= np.abs(kv4.E4M3 - want).min() * (1 + 1e-12)
            got = kv4.e2m1_value(codes[r, 16 * b:16 * b + 16]) * s
            best = np.abs(blk[:, None] - kv4.e2m1_value(np.arange(16)) * s).min(1)
            assert (np.abs(blk - got) <= best * (1 + 1e-12)).all()


def test_quantiser_edges():
    z = np.zeros(128)
    codes, scales = kv4.quantise(z, 0)
    assert not codes.any() and (scales == 1).all()
    x = z.copy()
    x[0], x[17], x[40] = np.inf, np.nan, -1e30
    codes, scales = kv4.quantise(x, 0)
    assert scales.tolist() == [0x7E, 0x7F, 0x7E, 1, 1, 1, 1, 1]
    assert codes[0] == 7 and codes[40] == 15 and not codes[16:32].any()
    assert np.isnan(kv4.values(codes, scales, 0)[16:32]).all()
    # ties go to the even code: with scale 1 (a 6 in the block), the midpoints
    x = z.copy()
    x[:8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]
    codes, scales = kv4.quantise(x, 0)
    assert scales[0] == 0x38 and codes[:8].tolist() == [7, 0, 2, 2, 4, 4, 6, 6]
    # a tie between two scales: 6 * 1.0625 lies between 6 * 1 and 6 * 1.125
    x = z.copy()
    x[3] = 6 * 1.0625
    assert kv4.quantise(x, 0)[1][0] == 0x38
    x[3] = 6 * 1.1875
    assert kv4.quantise(x, 0)[1][0] == 0x3A


def test_quantiser_scales_with_the_exponent():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(8, 128))
    a, b = kv4.quantise(x, 0), kv4.quantise(x * 2.0 ** 9, 9)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_layout_round_trip_and_places():
    rng = np.random.default_rng(2)
    kc, vc = (rng.integers(0, 16, size=(2, 3, 32, 128)).astype(np.uint8) for _ in range(2))
    ks, vs = (rng.integers(0, 256, size=(2, 3, 32, 8)).astype(np.uint8) for _ in range(2))
    cache = kv4.pack(kc, ks, vc, vs)
    assert cache.shape == (2, 3, 2, 2304)
    for a, b in zip(kv4.unpack(cache), (kc, ks, vc, vs)):
        assert np.array_equal(a, b)
    g = cache[1, 2, 1]  # tokens 16..31 of page 1, head 2
    assert g[2 * 256 + 5 * 16 + 3] == kc[1, 2, 21, 70] | kc[1, 2, 21, 71] << 4
    assert g[1024 + 7] == vc[1, 2, 16, 14] | vc[1, 2, 16, 15] << 4
    assert g[2048 + 15 * 8 + 7] == ks[1, 2, 31, 7] and g[2176 + 8] == vs[1, 2, 17, 0]


def test_extend_by_hand():
    lens, table, count, start, slots, caches, pos = kv4.extend([3, 4, 0], [2, 0, 5], [[7, -1, -1], [5, -1, -1], [-1, -1, -1]],
                                                               [9, 8, 2, 4], 4, 4, 9)
    assert lens.tolist() == [5, 4, 5] and count == 1 and start.tolist() == [0, 2, 2, 7]
    assert table.tolist() == [[7, 4, -1], [5, -1, -1], [2, 8, -1]]
    assert slots.tolist() == [31, 16, 8, 9, 10, 11, 32, -1, -1]
    assert caches.tolist() == [0, 0, 2, 2, 2, 2, 2, -1, -1] and pos.tolist() == [3, 4, 0, 1, 2, 3, 4, -1, -1]
    assert kv4.extend([0], [9], [[0, 0]], [1, 2, 3], 3, 4, 9) is None      # the row is full
    assert kv4.extend([0], [9], [[0, 0, 0]], [1, 2], 2, 4, 9) is None      # too few pages
    assert kv4.extend([0], [9], [[0, 0, 0]], [1, 2, 3], 3, 4, 8) is None   # too many tokens


def test_window_mask_by_hand():
    lines = kv4.node_lines([-1, 0, 0, 2], 4)
    assert [len(x) for x in lines] == [1, 2, 2, 3]
    assert kv4.visible(6, lines, 3, 0, 0) == (list(range(6)), [3, 2, 0])
    assert kv4.visible(6, lines, 3, 4, 2) == ([0, 1, 5], [3, 2, 0])   # position 8 sees 5..8 and 0, 1
    assert kv4.visible(6, lines, 3, 2, 0) == ([], [3, 2])
    assert kv4.visible(6, lines, 0, 1, 0) == ([], [0])
    assert kv4.visible(0, lines, 3, 1, 1) == ([], [3, 0])             # draft node 0 is the first token


def test_attention_without_window_is_the_draft_attention_oracle(oracle_mod):
    """Same numbers as the C++ oracle on the decoded (bf16) cache."""
    from paper_2604_26412_gb300 import workloads as wl
    rng = np.random.default_rng(3)
    hq, hkv, length, n, nq = 4, 2, 37, 5, 3
    parent = np.array([-1, 0, 0, 1, 3], np.int32)
    codes = [rng.integers(0, 16, size=(hkv, length, 128)) for _ in range(2)]
    scales = [rng.integers(40, 70, size=(hkv, length, 8)).astype(np.uint8) for _ in range(2)]
    pk, pv = (kv4.values(c, s, 0) for c, s in zip(codes, scales))
    q, dk, dv = (torch.from_numpy(rng.normal(size=s)).to(torch.bfloat16) for s in ((nq, hq, 128), (hkv, n, 128), (hkv, n, 128)))
    out, lse = kv4.attn(q.double().numpy(), pk, pv, dk.double().numpy(), dv.double().numpy(), parent, 0, 0, 128 ** -0.5)
    d = oracle_mod.make_desc(num_caches=1, num_seqs=1, hq=hq, hkv=hkv, head_dim=128, n_nodes=n, n_query=nq, n_max=n,
                             tree=True, l_cap=length)
    bits = lambda x: wl.bf16_bits(torch.as_tensor(x).to(torch.bfloat16)[None].contiguous())  # noqa: E731
    o2, l2 = oracle_mod.attn(d, bits(q), bits(pk), bits(pv), None, np.array([length], np.int32), bits(dk), bits(dv),
                             parent[None])
    assert np.abs(out - o2[0]).max() < 1e-12 and np.abs(lse - l2[0]).max() < 1e-12
