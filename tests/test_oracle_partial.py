"""Pins of the fp64 definitions of drafting over a part of a long cache (oracle/partial.py): closed forms, other ways to the
same numbers, and hand-made cases."""
import numpy as np
import pytest
import torch

from oracle import partial

D = 8


def pool(lens, page, hkv, seed=0):
    rng = np.random.default_rng(seed)
    used = [-(-n // page) for n in lens]
    ids = rng.permutation(sum(used) + 2)
    table = np.full((len(lens), max(used) + 1), -1)
    at = 0
    for c, u in enumerate(used):
        table[c, :u] = ids[at:at + u]
        at += u
    shape = (len(ids), hkv, page, D)
    return rng.standard_normal(shape), rng.standard_normal(shape), table


def test_bounds_by_hand_and_of_new_pages_alone():
    k = np.zeros((3, 1, 2, D))
    k[1, 0, 0, 0], k[1, 0, 1, 0], k[0, 0, 0, 0], k[0, 0, 1, 0] = 3, -1, 5, 99
    out = np.full((3, 1, 2, D), 7.0)
    got = partial.page_bounds(k, np.array([[1, 0]]), [3], [0], out)
    assert got[1, 0, :, 0].tolist() == [-1, 3] and got[0, 0, :, 0].tolist() == [5, 5]  # (the last token is past the length)
    assert (got[2] == 7).all()
    assert (partial.page_bounds(k, np.array([[1, 0]]), [3], [2], out)[1] == 7).all()


def test_scores_bound_the_keys_and_meet_them_where_a_page_is_one_token():
    for page in (1, 4):
        k, _, table = pool([13], page, 2)
        b = partial.page_bounds(k, table, [13], [0], np.zeros((len(k), 2, 2, D)))
        q = np.random.default_rng(1).standard_normal((1, 3, 6, D))
        got, mag = partial.page_scores(q, b, table, [13], page, 0.5, np.zeros((1, 3, 2, table.shape[1])))
        for h in range(2):
            s = 0.5 * np.einsum("ngd,jd->ngj", q[0, :, 3 * h:3 * h + 3], partial.rows_of(k, table, 0, 13, h)).max(1)
            best = np.stack([s[:, p * page:(p + 1) * page].max(1) for p in range(-(-13 // page))], axis=1)
            assert np.all(got[0, :, h, :best.shape[1]] >= best - 1e-12)
            if page == 1:
                assert np.allclose(got[0, :, h, :13], best, atol=1e-12)
        assert np.all(mag + 1e-12 >= np.abs(got))


@pytest.mark.parametrize("n,keep,first,last", [(1, 3, 0, 0), (9, 4, 0, 0), (9, 4, 1, 3), (9, 9, 0, 0), (40, 11, 2, 3)])
def test_selection_against_a_sort(n, keep, first, last):
    rng = np.random.default_rng(n)
    s = np.round(rng.standard_normal((5, n)), 1)
    picks, counts = partial.select_top(s, [n] * 5, 1, 1, keep, first, last)
    for r in range(5):
        i = np.arange(n)
        forced = (i < first) | (i >= n - last)
        want = np.sort(np.lexsort((i, -s[r], ~forced))[:min(n, keep)])
        assert counts[r] == len(want) and picks[r, :len(want)].tolist() == want.tolist() and (picks[r, len(want):] == -1).all()


def test_selection_ties_nan_and_shared_lengths():
    s = np.array([[1.0, np.nan, 1.0, 2.0, 0.0, -0.0], [5.0, 4.0, 3.0, 2.0, 1.0, 9.0]])
    assert partial.select_top(s[:1], [6], 1, 1, 3, 0, 0)[0].tolist() == [[0, 1, 3]]
    assert partial.select_top(s, [17], 2, 4, 2, 0, 1)[0].tolist() == [[1, 4], [0, 4]]  # (five entries: 17 tokens by 4)
    assert partial.select_top(s, [0], 2, 4, 2, 0, 1)[1].tolist() == [0, 0]


def test_attention_over_all_pages_is_the_causal_one():
    n, N = 11, 3
    k, v, table = pool([n], 4, 2)
    rng = np.random.default_rng(2)
    q, dk, dv = rng.standard_normal((1, N, 4, D)), rng.standard_normal((1, 2, N, D)), rng.standard_normal((1, 2, N, D))
    picks = np.broadcast_to(np.arange(3), (1, N, 2, 3))
    out, lse, spread, mag = partial.attn_sparse(q, k, v, table, [n], picks, np.full((1, N, 2), 3), dk, dv, None, 1, N, 0.3)
    for h in range(4):
        ks = torch.from_numpy(np.concatenate([partial.rows_of(k, table, 0, n, h // 2), dk[0, h // 2]]))
        vs = torch.from_numpy(np.concatenate([partial.rows_of(v, table, 0, n, h // 2), dv[0, h // 2]]))
        mask = torch.ones(N, n + N, dtype=torch.bool).tril(n)
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[0, :, h])[None], ks[None], vs[None],
                                                                attn_mask=mask, scale=0.3)[0]
        assert np.allclose(out[0, :, h], want.numpy(), atol=1e-12)
    assert np.all(spread >= np.abs(out) - 1e-12) and np.all(mag > 0)


def test_attention_over_no_page_or_one_and_of_a_tree():
    k, v, table = pool([8], 4, 1)
    q, dk, dv = np.zeros((1, 2, 1, D)), np.zeros((1, 1, 3, D)), np.arange(3.0)[None, None, :, None] * np.ones(D)
    parent = np.array([[-1, -1, 0]])
    args = (dk, dv, parent, 1, 3, 1.0)
    none, lse, _, _ = partial.attn_sparse(q, k, v, table, [8], np.zeros((1, 2, 1, 2), int), np.zeros((1, 2, 1), int), *args)
    assert np.allclose(none[0, 0], 1) and np.allclose(none[0, 1], 1)  # node 1 alone; nodes 2 and 0
    assert np.allclose(lse[0, :, 0], np.log([1, 2]))
    one, lse, _, _ = partial.attn_sparse(q, k, v, table, [6], np.ones((1, 2, 1, 2), int), np.ones((1, 2, 1), int), *args)
    assert np.allclose(lse[0, :, 0], np.log([3, 4]))                   # two tokens of the second page are below the length
    assert np.allclose(one[0, 0, 0], (v[table[0, 1], 0, :2].sum(0) + 1) / 3)


def test_weights_sum_to_the_rows_and_decay():
    k, _, table = pool([9, 0], 4, 2)
    rng = np.random.default_rng(3)
    q = rng.standard_normal((2, 2, 4, D))
    s = np.stack([[0.4 * partial.rows_of(k, table, 0, 9, h // 2) @ q[0, r, h] for h in range(4)] for r in range(2)])
    lse = np.zeros((2, 2, 4))
    lse[0] = np.log(np.exp(s).sum(-1))
    before = np.ones((2, 12))
    out, _ = partial.key_weights(q, k, table, [9, 0], lse, 0.5, before, np.full((2, 12), 7.0), 0.4)
    assert np.isclose(out[0, :9].sum(), 9 * 0.5 + 8) and (out[0, 9:] == 7).all() and (out[1] == 7).all()
    lse[0, 1] = -np.inf
    out, _ = partial.key_weights(q, k, table, [9, 0], lse, 0.0, before, np.full((2, 12), 7.0), 0.4)
    assert np.isclose(out[0, :9].sum(), 4)


def test_eviction_by_hand():
    k = np.arange(24.0).reshape(6, 1, 4, 1)
    table = np.array([[2, 0, 5], [1, 3, -1]])
    kept, counts = np.array([[1, 4, 9], [0, 1, 2]]), [3, 3]
    w = np.arange(20.0).reshape(2, 10)
    out = partial.cache_evict(k, -k, table, [10, 5], kept, counts, w, k, -k, table, w, np.full(6, -1), 1)
    assert out[0][2, 0, :3, 0].tolist() == [9, 0, 21] and out[0][2, 0, 3, 0] == 11  # (slots past the last one stay)
    assert out[0][1, 0, :, 0].tolist() == [4, 5, 6, 7] and np.array_equal(out[1], -out[0])
    assert out[2].tolist() == [3, 3] and out[3][0].tolist() == [1, 4, 9] + 7 * [0] and out[3][1, :3].tolist() == [10, 11, 12]
    assert out[4].tolist() == [-1, 0, 5, 3, -1, -1] and out[5] == 4
