"""Refusals of the 4-bit cache's entry points, on the CPU: every bad argument has its status code before anything is
enqueued; the Python descriptors mirror the C structs."""
import ctypes
import os
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


@pytest.mark.parametrize("struct,cls", [("kvshot_extend_desc", kvshot.ExtendDesc), ("kvshot_kv4_desc", kvshot.Kv4Desc)])
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


def _extend(ptrs=None, **kw):
    d = dict(num_caches=4, page_size=16, max_pages_per_seq=8, num_pages=64, max_tokens=32)
    d.update(kw)
    names = ["seq_lens", "new_tokens", "page_table", "free_pages", "free_count", "seq_lens_out", "page_table_out",
             "free_count_out", "token_start", "slots", "token_cache", "positions"]
    p = {n: A for n in names} | (ptrs or {})
    return kvshot.cache_extend_status(kvshot.make_extend_desc(**d), *[p[n] for n in names], stream=0)


@pytest.mark.parametrize("kw,code", [
    (dict(num_caches=0), SHAPE), (dict(num_caches=1025), UNSUPPORTED), (dict(page_size=0), SHAPE),
    (dict(max_pages_per_seq=0), SHAPE), (dict(num_pages=0), SHAPE), (dict(max_tokens=-1), SHAPE),
    (dict(num_free=-1), SHAPE), (dict(max_pages_per_seq=1 << 28), UNSUPPORTED), (dict(num_pages=1 << 28), UNSUPPORTED),
])
def test_extend_sizes(kw, code):
    assert _extend(**kw) == code


@pytest.mark.parametrize("name", ["seq_lens", "new_tokens", "page_table", "free_pages", "free_count", "seq_lens_out",
                                  "page_table_out", "free_count_out", "token_start"])
def test_extend_pointers(name):
    assert _extend({name: None}) == NULL
    assert _extend({name: A + 2}) == ALIGN


def test_extend_maps_are_checked_for_alignment():
    for name in ("slots", "token_cache", "positions"):
        assert _extend({name: A + 1}) == ALIGN
    assert kvshot.cache_extend_status(None, *[A] * 12, stream=0) == NULL


def _rows(call, ptrs=None, **kw):
    d = dict(num_tokens=4, hkv=8, page_size=16, num_pages=4)
    d.update(kw)
    p = dict(k=A, v=A, slots=A, cache=A) | (ptrs or {})
    desc = kvshot.make_kv4_desc(**d)
    if call == "store":
        return kvshot.kv4_store_status(desc, p["k"], p["v"], p["slots"], p["cache"], stream=0)
    return kvshot.kv4_load_status(desc, p["cache"], p["slots"], p["k"], p["v"], stream=0)


@pytest.mark.parametrize("call", ["store", "load"])
@pytest.mark.parametrize("kw,code", [
    (dict(num_tokens=-1), SHAPE), (dict(hkv=0), SHAPE), (dict(head_dim=64), UNSUPPORTED), (dict(page_size=0), SHAPE),
    (dict(page_size=8), UNSUPPORTED), (dict(page_size=24), UNSUPPORTED), (dict(num_pages=0), SHAPE),
    (dict(num_pages=1 << 24, page_size=256), UNSUPPORTED), (dict(k_scale_exp=65), SHAPE), (dict(v_scale_exp=-65), SHAPE),
    (dict(k_scale_exp=-2 ** 31), SHAPE), (dict(k_stride=1016), SHAPE), (dict(v_stride=1028), ALIGN),
    (dict(k_stride=1 << 62), SHAPE), (dict(num_tokens=0), OK),
])
def test_row_sizes(call, kw, code):
    assert _rows(call, **kw) == code


@pytest.mark.parametrize("call", ["store", "load"])
def test_row_pointers(call):
    for name in ("k", "v", "slots", "cache"):
        assert _rows(call, {name: None}) == NULL
        assert _rows(call, {name: A + 2}) == ALIGN
    assert _rows(call, {"k": A + 8}) == ALIGN


def test_cache_bytes():
    assert kvshot.kv4_cache_bytes(3, 8, 32) == 3 * 8 * 2 * 2304
    assert kvshot.kv4_cache_bytes(1 << 20, 8, 128) == (1 << 20) * 8 * 8 * 2304  # beyond 32 bits
    for bad in ((0, 8, 16), (1, 0, 16), (1, 8, 0), (1, 8, 20), (1 << 24, 8, 16)):
        assert kvshot.kv4_cache_bytes(*bad) == 0


def _attn(ptrs=None, window=0, sinks=0, ws=(A, 1 << 40), **kw):
    base = dict(num_caches=2, num_seqs=2, hq=32, hkv=8, n_nodes=8, n_query=4, n_max=8, max_seq_len=64,
                page_size=16, max_pages_per_seq=4, num_pages=8, l_cap=64, tree=True)
    base.update(kw)
    d = kvshot.make_desc(**base, workspace=ws[0], workspace_bytes=ws[1])
    p = dict(q=A, cache=A, pt=A, sl=A, dk=A, dv=A, par=A, out=2 * A, lse=3 * A) | (ptrs or {})
    return kvshot.draft_attn_kv4_status(d, p["q"], p["cache"], p["pt"], p["sl"], p["dk"], p["dv"], p["par"], window,
                                        sinks, p["out"], p["lse"], stream=0)


@pytest.mark.parametrize("kw,code", [
    (dict(num_caches=0), SHAPE), (dict(num_caches=2048, num_seqs=2048), UNSUPPORTED), (dict(hq=30), SHAPE),
    (dict(head_dim=64), UNSUPPORTED), (dict(n_query=9), SHAPE), (dict(n_nodes=9), SHAPE),
    (dict(n_nodes=65, n_max=80), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=40), UNSUPPORTED),
    (dict(page_size=0), SHAPE), (dict(num_pages=0), SHAPE), (dict(max_pages_per_seq=0), SHAPE),
    (dict(max_seq_len=-1), SHAPE), (dict(flags=0x80), SHAPE), (dict(flags=kvshot.KVSHOT_TARGET_FP8), UNSUPPORTED),
    (dict(flags=kvshot.KVSHOT_FORCE_TC), UNSUPPORTED), (dict(flags=kvshot.KVSHOT_FORCE_MMA), UNSUPPORTED),
    (dict(flags=kvshot.KVSHOT_FORCE_CC), UNSUPPORTED), (dict(k_scale_exp=65), SHAPE), (dict(v_scale_exp=-65), SHAPE),
    (dict(window=-1), SHAPE), (dict(sinks=-1), SHAPE), (dict(scale=-1.0), SHAPE), (dict(num_ctas=-1), SHAPE),
    (dict(ptrs=dict(pt=None), l_cap=72), UNSUPPORTED), (dict(ptrs=dict(pt=None), l_cap=0), SHAPE),
    (dict(n_query=0), OK),
])
def test_attn_sizes(kw, code):
    assert _attn(**kw) == code


def test_attn_pointers():
    for name in ("q", "cache", "sl", "dk", "dv", "par", "out", "lse"):
        assert _attn({name: None}) == NULL
        assert _attn({name: A + 2}) == ALIGN
    assert _attn({"pt": A + 2}) == ALIGN
    assert kvshot.draft_attn_kv4_workspace_size(kvshot.make_desc(
        num_caches=2, num_seqs=2, hq=30, hkv=8, n_nodes=8, n_query=4, n_max=8, max_seq_len=64)) == 0
