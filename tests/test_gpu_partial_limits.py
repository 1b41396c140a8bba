"""Lengths that have no room at all are recorded by every entry point that looks at them."""
import pytest
import torch

from paper_2604_26412_gb300 import kvshot

from .partial_problems import D, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,code", [([0, 0], 0), ([0, 5], kvshot.KVSHOT_ERR_DEVICE_BOUNDS), ([-1, 0], kvshot.KVSHOT_ERR_DEVICE_BOUNDS)])
def test_lengths_without_room_are_looked_at(lens, code):
    p = Problem([20, 40], 16, nodes=2, query=2)
    p.desc.max_seq_len = 0
    p.t_lens.copy_(p.ints(lens))
    bounds = torch.full((p.num_pages, 8, 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
    scores = torch.full((2, 2, 8, p.table.shape[1]), 7.0, device="cuda")
    w = torch.full((2, 50), 7.0, device="cuda")
    picks, counts = torch.zeros((2, 2, 8, 4), dtype=torch.int32, device="cuda"), torch.zeros((2, 2, 8), dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(p.q), torch.empty((2, 2, 32), device="cuda")
    ws = p.workspace(4)
    for call in (lambda: kvshot.page_bounds(p.desc, p.k, p.t_table, p.t_lens, None, bounds),
                 lambda: kvshot.page_bounds(p.desc, p.k, p.t_table, p.t_lens, p.ints([0, 3]), bounds),
                 lambda: kvshot.page_scores(p.desc, p.q, bounds, p.t_table, p.t_lens, scores),
                 lambda: kvshot.draft_attn_sparse(p.desc, p.q, p.k, p.v, p.t_table, p.t_lens, picks, counts, 4, p.dk, p.dv, None, out, lse),
                 lambda: kvshot.key_weights(p.desc, p.q, p.k, p.t_table, p.t_lens, lse, 1.0, 50, w, w)):
        call()
        torch.cuda.synchronize()
        assert int(p.err.item()) == code
        p.err.zero_()
    del ws
    assert all(bool((x == 7).all()) for x in (bounds, scores, w))


@pytest.mark.parametrize("hq", [0, 8])
def test_bounds_need_no_query_heads(hq):
    p = Problem([20, 300], 16, hq=8, hkv=8)
    want, got = (torch.full((p.num_pages, 8, 2, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kvshot.page_bounds(p.desc, p.k, p.t_table, p.t_lens, None, want)
    p.desc.hq, p.desc.n_nodes, p.desc.n_query, p.desc.n_max, p.desc.scale = hq, 0, 0, 0, 0.0
    kvshot.page_bounds(p.desc, p.k, p.t_table, p.t_lens, None, got)
    torch.cuda.synchronize()
    assert int(p.err.item()) == 0 and torch.equal(want, got)
