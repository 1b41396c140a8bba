"""Every entry point as the first CUDA call of a host thread, which has no context current yet.

The library's functions are replaced by ones that run each call in a thread of its own; results are those of calls from the
main thread, bit for bit.
"""
import threading

import pytest
import torch

from paper_2604_26412_gb300 import kv4, kvshot
from paper_2604_26412_gb300 import workloads as wl
from paper_2604_26412_gb300.partial import PageSelection, TokenWeights
from paper_2604_26412_gb300.step import DraftStep

from .partial_problems import Problem
from .test_gpu_partial_streams import calls

pytestmark = pytest.mark.gpu


class FreshThreads:
    def __init__(self, lib):
        self.lib, self.called = lib, set()

    def __getattr__(self, name):
        f = getattr(self.lib, name)

        def call(*args):
            got = []
            self.called.add(name)
            t = threading.Thread(target=lambda: got.append(f(*args)))
            t.start()
            t.join()
            return got[0]
        return call


def step(levels, mode="per_depth", page=16, lens=(300, 40, 700), fp8=False, kv4_cache=False, norm=False, pages=False,
         weights=False, hq=32, hkv=8, **kw):
    def make():
        spec = wl.Spec("threads", len(lens), 1, list(lens), list(levels), len(levels) > 1, True, page_size=page, hq=hq, hkv=hkv, seed=4)
        inp = wl.make_inputs(spec, "cuda", seed=4)
        w = TokenWeights(inp) if weights else None
        if fp8:
            kw["target_fp8"] = (*wl.fp8_target(inp), wl.FP8_K_EXP, wl.FP8_V_EXP)
        if kv4_cache:
            kw["target_kv4"] = kv4.of_inputs(inp)
            kw["target_kv4"].values(kw["target_kv4"].slots)
        if norm:
            one = torch.ones(128, dtype=torch.bfloat16, device="cuda")
            kw["qk_norm"] = (one, one, 1e-6)
        s = DraftStep(inp, mode, pages=PageSelection(inp, keep=20) if pages else None, weights=w, **kw)
        s.run()
        if w is not None:
            w.evict(100)
        torch.cuda.synchronize()
        assert s.error_code() == 0
        return [*s.out, *s.lse, inp.seq_lens, *([w.weights] if w is not None else [])]
    return make


def fusion():
    fi = wl.fusion_inputs(33, 256, device="cuda", seed=1)
    d = kvshot.make_fusion_desc(num_tokens=33, hidden=256)
    ws = torch.empty(kvshot.gated_delta_workspace_size(d), dtype=torch.uint8, device="cuda")
    d.workspace, d.workspace_bytes = ws.data_ptr(), ws.numel()
    h = torch.empty_like(fi.n)
    kvshot.gated_delta(d, fi.n, fi.o, fi.w_g, fi.b_g, fi.w_delta, h)
    torch.cuda.synchronize()
    return [h]


def projection():
    pi = wl.project_inputs(33, 3, 2, device="cuda", seed=1)
    d = kvshot.make_project_desc(num_tokens=33, num_layers=3, hkv=2, num_caches=1, l_cap=33)
    ws = torch.empty(kvshot.kv_project_workspace_size(d), dtype=torch.uint8, device="cuda")
    d.workspace, d.workspace_bytes = ws.data_ptr(), ws.numel()
    out = [torch.zeros((66, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    zeros, place = torch.zeros(33, dtype=torch.int32, device="cuda"), torch.arange(33, dtype=torch.int32, device="cuda")
    kvshot.kv_project(d, pi.k_in, pi.v_in, pi.w_k, pi.w_v, zeros, place, None, *out)
    torch.cuda.synchronize()
    return out


def partial_calls(**problem):
    def make():
        p = Problem(**problem)
        run, o = calls(p)
        run()
        torch.cuda.synchronize()
        assert int(p.err.item()) == 0
        return list(o.values())
    return make


FLOWS = {
    "mma": step((1,)), "tcgen05": step((12,)), "whole": step((8, 28, 28), "whole"), "CUDA cores": step((1,), flags=kvshot.KVSHOT_FORCE_CC),
    "fp8": step((1,), fp8=True), "fp8 tcgen05": step((12,), fp8=True), "4 bits": step((1,), kv4_cache=True),
    "4 bits, many rows": step((12,), kv4_cache=True), "norm": step((2,), norm=True), "fusion": fusion, "projection": projection,
    "pages": step((3, 12), pages=True), "weights": step((12, 24), weights=True),
    "partial": partial_calls(lens=[300, 0, 65], page=16, nodes=3, query=2, seed=5),
    "partial, large": partial_calls(lens=[300, 9001, 700, 64, 65, 128, 500, 33, 31, 900, 1000, 77, 90], page=16, nodes=12, query=12,
                                    tree=True, seed=3),
}


@pytest.mark.parametrize("name", FLOWS)
def test_first_calls_of_threads(monkeypatch, name):
    want = FLOWS[name]()
    fresh = FreshThreads(kvshot.load())
    monkeypatch.setattr(kvshot, "_lib", fresh)
    got = FLOWS[name]()
    assert fresh.called
    assert all(torch.equal(x.contiguous().view(torch.int16), y.contiguous().view(torch.int16)) for x, y in zip(got, want))
