"""Refusals of the entry points that draft over a part of a long cache, on the CPU: every bad argument has its status code
before anything is enqueued; the Python descriptors mirror the C structs."""
import ctypes
import subprocess

import pytest

from paper_2604_26412_gb300 import build as kbuild
from paper_2604_26412_gb300 import kvshot

A = 1 << 20  # a fake, aligned device address: every case below fails before it is used
OK, NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = (
    kvshot.KVSHOT_OK, kvshot.KVSHOT_ERR_NULL, kvshot.KVSHOT_ERR_SHAPE, kvshot.KVSHOT_ERR_ALIGN,
    kvshot.KVSHOT_ERR_UNSUPPORTED, kvshot.KVSHOT_ERR_WORKSPACE)


@pytest.fixture(scope="module", autouse=True)
def lib():
    kbuild.build()
    return kvshot.load()


@pytest.mark.parametrize("struct,cls", [("kvshot_select_desc", kvshot.SelectDesc), ("kvshot_evict_desc", kvshot.EvictDesc)])
def test_descriptors_mirror_the_header(tmp_path, struct, cls):
    fields = [f for f, _ in cls._fields_]
    src = ["#include <stdio.h>", "#include <stddef.h>", '#include "kvshot.h"', "int main(void) {",
           f'printf("%zu\\n", sizeof({struct}));', *[f'printf("%zu\\n", offsetof({struct}, {f}));' for f in fields],
           "return 0; }"]
    (tmp_path / "a.c").write_text("\n".join(src))
    subprocess.run(["gcc", "-I", kbuild.INCLUDE, str(tmp_path / "a.c"), "-o", str(tmp_path / "a")], check=True)
    vals = [int(v) for v in subprocess.run([str(tmp_path / "a")], capture_output=True, text=True).stdout.split()]
    assert vals[0] == ctypes.sizeof(cls)
    assert vals[1:] == [getattr(cls, f).offset for f in fields]


def _desc(ws=(A, 1 << 40), **kw):
    base = dict(num_caches=2, num_seqs=2, hq=32, hkv=8, n_nodes=8, n_query=4, n_max=8, max_seq_len=64, page_size=16,
                max_pages_per_seq=4, num_pages=8, l_cap=64)
    base.update(kw)
    return kvshot.make_desc(**base, workspace=ws[0], workspace_bytes=ws[1])


def bounds(ptrs=None, **kw):
    p = dict(k=A, pt=A, sl=A, fr=A, out=A) | (ptrs or {})
    return kvshot.page_bounds_status(_desc(**kw), p["k"], p["pt"], p["sl"], p["fr"], p["out"], stream=0)


def scores(ptrs=None, **kw):
    p = dict(q=A, b=A, pt=A, sl=A, out=A) | (ptrs or {})
    return kvshot.page_scores_status(_desc(**kw), p["q"], p["b"], p["pt"], p["sl"], p["out"], stream=0)


def sparse(ptrs=None, max_picks=4, ws=(A, 1 << 40), **kw):
    p = dict(q=A, k=A, v=A, pt=A, sl=A, pk=A, ct=A, dk=A, dv=A, par=A, out=A, lse=A) | (ptrs or {})
    return kvshot.draft_attn_sparse_status(_desc(ws, **kw), p["q"], p["k"], p["v"], p["pt"], p["sl"], p["pk"], p["ct"],
                                           max_picks, p["dk"], p["dv"], p["par"], p["out"], p["lse"], stream=0)


def weights(ptrs=None, decay=1.0, width=64, **kw):
    p = dict(q=A, k=A, pt=A, sl=A, lse=A, w=A, out=A) | (ptrs or {})
    return kvshot.key_weights_status(_desc(**kw), p["q"], p["k"], p["pt"], p["sl"], p["lse"], decay, width, p["w"], p["out"],
                                     stream=0)


BAD_DESC = [
    (dict(num_caches=0), SHAPE), (dict(num_caches=2048, num_seqs=2048), UNSUPPORTED), (dict(num_caches=3), SHAPE),
    (dict(hq=30), SHAPE), (dict(hq=33 * 8), UNSUPPORTED), (dict(head_dim=64), UNSUPPORTED), (dict(n_query=9), SHAPE),
    (dict(n_nodes=9), SHAPE), (dict(page_size=12), UNSUPPORTED), (dict(page_size=0), UNSUPPORTED),
    (dict(page_size=512), UNSUPPORTED), (dict(num_pages=0), SHAPE), (dict(max_pages_per_seq=0), SHAPE),
    (dict(num_pages=1 << 28), UNSUPPORTED), (dict(max_pages_per_seq=1 << 30), UNSUPPORTED), (dict(max_seq_len=-1), SHAPE),
    (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(flags=0x80), SHAPE),
    (dict(flags=kvshot.KVSHOT_TARGET_FP8), UNSUPPORTED), (dict(flags=kvshot.KVSHOT_FORCE_TC), UNSUPPORTED),
    (dict(flags=kvshot.KVSHOT_FORCE_MMA), UNSUPPORTED), (dict(flags=kvshot.KVSHOT_FORCE_CC), UNSUPPORTED),
    (dict(n_nodes=1 << 26, n_query=1 << 26, n_max=1 << 26), UNSUPPORTED),
    (dict(max_pages_per_seq=1 << 27, max_seq_len=2 ** 31 - 1), UNSUPPORTED),
]


@pytest.mark.parametrize("call", [bounds, scores, sparse, weights])
@pytest.mark.parametrize("kw,code", BAD_DESC)
def test_descriptors(call, kw, code):
    assert call(**kw) == code


def test_null_descriptors():
    assert kvshot.page_bounds_status(None, A, A, A, A, A, stream=0) == NULL
    assert kvshot.page_scores_status(None, A, A, A, A, A, stream=0) == NULL
    assert kvshot.select_top_status(None, A, A, A, A, stream=0) == NULL
    assert kvshot.draft_attn_sparse_status(None, A, A, A, A, A, A, A, 4, A, A, A, A, A, stream=0) == NULL
    assert kvshot.key_weights_status(None, A, A, A, A, A, 1.0, 4, A, A, stream=0) == NULL
    assert kvshot.cache_evict_status(None, *[A] * 15, stream=0) == NULL
    assert kvshot.draft_attn_sparse_workspace_size(None, 4) == 0


@pytest.mark.parametrize("call,names,wide", [
    (bounds, ["k", "pt", "sl", "out"], ["k", "out"]), (scores, ["q", "b", "pt", "sl", "out"], ["q", "b"]),
    (sparse, ["q", "k", "v", "pt", "sl", "pk", "ct", "dk", "dv", "out", "lse"], ["q", "k", "v", "dk", "dv", "out"]),
    (weights, ["q", "k", "sl", "lse", "out"], ["q", "k"]),
])
def test_pointers(call, names, wide):
    for name in names:
        assert call({name: None}) == NULL
        assert call({name: A + 2}) == ALIGN
    for name in wide:
        assert call({name: A + 8}) == ALIGN
    if call is scores:
        assert call({"b": A + 16}) == ALIGN
    if call is sparse:
        for name in ("k", "v", "dk", "dv"):
            assert call({name: A + 16}) == ALIGN
    if call is bounds:
        assert call({"fr": A + 2}) == ALIGN
    if call is weights:
        assert call({"w": A + 2}) == ALIGN and call({"pt": A + 2}) == ALIGN


def test_calls_without_rows_do_nothing():
    assert scores({"q": None}, n_query=0) == OK
    assert sparse({"q": None}, n_query=0) == OK
    assert kvshot.select_top_status(kvshot.make_select_desc(num_rows=0, row_len=1, keep=1), None, None, None, None, stream=0) == OK


def test_sparse_workspace_and_lists():
    assert sparse(max_picks=0) == SHAPE
    assert sparse(max_picks=1 << 25) == UNSUPPORTED
    assert sparse(ws=(0, 1 << 40)) == WORKSPACE
    assert sparse(ws=(A + 128, 1 << 40)) == WORKSPACE
    need = kvshot.draft_attn_sparse_workspace_size(_desc(), 4)
    assert need > 0 and sparse(ws=(A, need - 1)) == WORKSPACE
    assert kvshot.draft_attn_sparse_workspace_size(_desc(hq=30), 4) == 0
    assert kvshot.draft_attn_sparse_workspace_size(_desc(), 0) == 0
    assert sparse({"par": None}, tree=True) == NULL
    assert sparse({"par": A + 2}, tree=True) == ALIGN
    assert sparse(tree=True, n_nodes=65, n_max=65) == UNSUPPORTED


def test_weights_numbers():
    for decay in (-0.1, 1.5, float("nan"), float("inf")):
        assert weights(decay=decay) == SHAPE
    assert weights(width=-1) == SHAPE
    assert weights({"pt": None}, l_cap=0) == SHAPE


@pytest.mark.parametrize("kw", [dict(num_rows=-1), dict(row_len=0), dict(rows_per_len=0), dict(rows_per_len=3),
                                dict(tokens_per_entry=0), dict(keep=0), dict(first=-1), dict(last=-1), dict(first=3, last=2),
                                dict(first=2 ** 31 - 1, last=2 ** 31 - 1)])
def test_select_sizes(kw):
    d = dict(num_rows=4, row_len=16, rows_per_len=2, tokens_per_entry=16, keep=4, first=1, last=1) | kw
    assert kvshot.select_top_status(kvshot.make_select_desc(**d), A, A, A, A, stream=0) == SHAPE


def test_select_sizes_beyond_its_numbers():
    for kw in (dict(row_len=2 ** 31 - 1), dict(keep=2 ** 31 - 1), dict(num_rows=2 ** 28)):
        d = dict(num_rows=4, row_len=16, keep=4) | kw
        assert kvshot.select_top_status(kvshot.make_select_desc(**d), A, A, A, A, stream=0) == UNSUPPORTED


def test_select_pointers():
    d = kvshot.make_select_desc(num_rows=4, row_len=16, keep=4)
    for i in range(4):
        assert kvshot.select_top_status(d, *[None if j == i else A for j in range(4)], stream=0) == NULL
        assert kvshot.select_top_status(d, *[A + 2 if j == i else A for j in range(4)], stream=0) == ALIGN


NAMES = ["k", "v", "pt", "sl", "kept", "count", "w", "k_out", "v_out", "pt_out", "sl_out", "w_out", "free", "fc", "fc_out"]


def evict(ptrs=None, **kw):
    d = dict(num_caches=2, hkv=8, page_size=16, max_pages_per_seq=4, num_pages=8, max_kept=32, weights_len=64)
    d.update(kw)
    p = {n: A for n in NAMES} | dict(k_out=2 * A, v_out=2 * A, pt_out=2 * A, w_out=2 * A) | (ptrs or {})
    return kvshot.cache_evict_status(kvshot.make_evict_desc(**d), *[p[n] for n in NAMES], stream=0)


@pytest.mark.parametrize("kw,code", [
    (dict(num_caches=0), SHAPE), (dict(num_caches=1025), UNSUPPORTED), (dict(hkv=0), SHAPE), (dict(hkv=20000), UNSUPPORTED),
    (dict(page_size=0), SHAPE), (dict(max_pages_per_seq=0), SHAPE), (dict(num_pages=0), SHAPE), (dict(max_pages_out=0), SHAPE),
    (dict(num_pages_out=0), SHAPE), (dict(max_kept=0), SHAPE), (dict(weights_len=-1), SHAPE), (dict(weights_len_out=-1), SHAPE),
    (dict(num_free=-1), SHAPE), (dict(num_pages=1 << 28), UNSUPPORTED), (dict(num_pages_out=1 << 28), UNSUPPORTED),
    (dict(head_dim=64), UNSUPPORTED), (dict(page_size=1 << 30), UNSUPPORTED), (dict(max_pages_per_seq=1 << 29), UNSUPPORTED),
    (dict(max_pages_out=1 << 29), UNSUPPORTED), (dict(max_kept=2 ** 31 - 1), UNSUPPORTED),
    (dict(weights_len=2 ** 31 - 1), UNSUPPORTED), (dict(weights_len_out=2 ** 31 - 1), UNSUPPORTED),
])
def test_evict_sizes(kw, code):
    assert evict(**kw) == code


def test_evict_pointers():
    for name in NAMES:
        if name in ("w", "w_out", "free", "fc", "fc_out"):
            assert evict({name: None}) == NULL  # (only all of them can be left out)
        else:
            assert evict({name: None}) == NULL
        assert evict({name: A + 2}) == ALIGN
    for name in ("k", "v", "k_out", "v_out"):
        assert evict({name: 3 * A + 8}) == ALIGN


def test_evict_in_place_is_all_or_nothing():
    assert evict({"k_out": A}) == SHAPE
    assert evict({"v_out": A}) == SHAPE
    assert evict({"k_out": A, "v_out": A}) == SHAPE
    assert evict({"k_out": A, "v_out": A, "pt_out": A}, max_pages_out=3) == SHAPE
    assert evict({"k_out": A, "v_out": A, "pt_out": A}, num_pages_out=7) == SHAPE
    assert evict({"w_out": A}, weights_len_out=32) == SHAPE
