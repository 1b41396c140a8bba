"""Draft attention and the KV projection from two host threads, each on a stream of its own with problems of its own size: the
limit of a kernel's shared memory is the process's, and one thread's calls must not take it from the other's."""
import threading

import pytest
import torch

from paper_2604_26412_gb300 import kvshot
from paper_2604_26412_gb300 import workloads as wl

from .partial_problems import D, Problem

pytestmark = pytest.mark.gpu

CALLS = 1500


def attention(caches, query, flags):
    """call(stream) and its outputs: a batch of short caches, of e4m3 codes with KVSHOT_TARGET_FP8."""
    p = Problem([70] * caches, 16, nodes=query, query=query, seed=caches)
    p.desc.flags |= flags
    k, v = p.k, p.v
    if flags & kvshot.KVSHOT_TARGET_FP8:
        g = torch.Generator("cuda").manual_seed(caches)
        k, v = (torch.randint(0, 0x60, x.shape, generator=g, dtype=torch.uint8, device="cuda") for x in (k, v))
    size = kvshot.workspace_size(p.desc)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    p.desc.workspace, p.desc.workspace_bytes = ws.data_ptr(), size
    table, out, lse = p.t_table.clamp(min=0), torch.zeros_like(p.q), torch.zeros(p.q.shape[:3], device="cuda")

    def call(stream):
        return kvshot.draft_attn_status(p.desc, p.q, k, v, table, p.t_lens, p.dk, p.dv, None, out, lse, stream)
    call.keep = ws
    return call, (out, lse), p.err


def projection(tokens, layers):
    pi = wl.project_inputs(tokens, layers, 2, device="cuda", seed=tokens)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    d = kvshot.make_project_desc(num_tokens=tokens, num_layers=layers, hkv=2, num_caches=1, l_cap=tokens, err_flag=err)
    ws = torch.empty(kvshot.kv_project_workspace_size(d), dtype=torch.uint8, device="cuda")
    d.workspace, d.workspace_bytes = ws.data_ptr(), ws.numel()
    cache, place = torch.zeros(tokens, dtype=torch.int32, device="cuda"), torch.arange(tokens, dtype=torch.int32, device="cuda")
    out = [torch.zeros((2 * tokens, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def call(stream):
        return kvshot.kv_project_status(d, pi.k_in, pi.v_in, pi.w_k, pi.w_v, cache, place, None, *out, stream)
    call.keep = ws
    return call, out, err


FP8 = kvshot.KVSHOT_TARGET_FP8
PAIRS = {
    "mma": lambda: [attention(c, 1, 0) for c in (2, 300)],
    "tcgen05": lambda: [attention(c, 12, 0) for c in (2, 300)],
    "paired rows": lambda: [attention(c, 64, 0) for c in (2, 300)],
    "CUDA cores": lambda: [attention(c, 1, kvshot.KVSHOT_FORCE_CC) for c in (2, 300)],
    "fp8 mma": lambda: [attention(c, 1, FP8) for c in (2, 300)],
    "fp8 tcgen05": lambda: [attention(c, 12, FP8) for c in (2, 300)],
    "projection": lambda: [projection(5, 1), projection(256, 4)],
}


@pytest.mark.parametrize("name", PAIRS)
def test_threads_with_problems_of_other_sizes(name):
    jobs = PAIRS[name]()
    streams = [torch.cuda.Stream() for _ in jobs]
    want = []
    for call, outs, _ in jobs:
        assert call(torch.cuda.current_stream()) == kvshot.KVSHOT_OK
        torch.cuda.synchronize()
        want.append([x.clone() for x in outs])
        for x in outs:
            x.zero_()
    torch.cuda.synchronize()
    start, refused = threading.Barrier(len(jobs)), []

    def work(call, handle):
        start.wait()
        for _ in range(CALLS):
            status = call(handle)
            if status != kvshot.KVSHOT_OK:
                refused.append(status)
    threads = [threading.Thread(target=work, args=(call, s.cuda_stream)) for (call, _, _), s in zip(jobs, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not refused, f"{len(refused)} of {CALLS * len(jobs)} calls refused: {refused[0]}"
    for (_, outs, err), expected in zip(jobs, want):
        assert int(err.item()) == 0
        assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(outs, expected))
