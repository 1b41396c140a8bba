"""The 4-bit cache attention's waits, as tests/test_gpu_watchdog.py drives the other kernels': with a limit of 1 ns a call
ends, records KVSHOT_ERR_TIMEOUT, and leaves everything fit for the next one, which gives what an unlimited call gives.
"""
import pytest
import torch

from paper_2604_26412_gb300 import kvshot
from tests.test_gpu_kv4 import D, _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,nodes", [(8, 2), (8, 4), (8, 8), (8, 12), (8, 16), (8, 40)])
def test_waits_that_run_out_are_recorded(hq, nodes):
    """8, 16, 32, 48, 64 and 160 rows over 8 contexts of 40000 tokens, whose 92 MB take every CTA many loads of a microsecond
    and more: with a limit of 1 ns some wait runs out, in each of four calls, and the next call is right."""
    c, length, hkv = 8, 40000, 2
    gen = torch.Generator("cuda").manual_seed(nodes)
    cache = torch.randint(0, 256, (c, hkv, length // 16, 2304), dtype=torch.uint8, device="cuda", generator=gen)
    cache[..., 2048:] = torch.randint(0x30, 0x40, (c, hkv, length // 16, 256), dtype=torch.uint8, device="cuda", generator=gen)
    bf = lambda *s: torch.randn(s, device="cuda", generator=gen).to(torch.bfloat16)  # noqa: E731
    q, dk, dv = bf(c, nodes, hq, D), bf(c, hkv, nodes, D), bf(c, hkv, nodes, D)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = kvshot.make_desc(num_caches=c, num_seqs=c, hq=hq, hkv=hkv, n_nodes=nodes, n_query=nodes, n_max=nodes,
                            max_seq_len=length, l_cap=length, err_flag=err)
    ws = torch.empty(kvshot.draft_attn_kv4_workspace_size(desc), dtype=torch.uint8, device="cuda")
    desc.workspace, desc.workspace_bytes = ws.data_ptr(), ws.numel()
    lens = _i32([length] * c)

    def run(limit):
        desc.wait_limit_ns = limit
        err.zero_()
        out, lse = torch.full_like(q, float("nan")), torch.full((c, nodes, hq), float("nan"), device="cuda")
        kvshot.draft_attn_kv4(desc, q, cache, None, lens, dk, dv, None, 0, 0, out, lse)
        return int(err.item()), out, lse

    code, out, lse = run(0)
    assert code == 0 and bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    for _ in range(4):
        assert run(1)[0] == kvshot.KVSHOT_ERR_TIMEOUT
        code, o, l = run(0)
        assert code == 0 and torch.equal(o, out) and torch.equal(l, lse)
