"""Page scores from several host threads, each on a stream of its own."""
import threading

import pytest
import torch

from paper_2604_26412_gb300 import kvshot

from .partial_problems import D, Problem

pytestmark = pytest.mark.gpu

CALLS = 2000
LENS = [0, 1, 1023, 1024, 1032, 5003] + [2049] * 30


def test_threads_that_score_levels_of_other_sizes():
    """48 and 64 columns of q: the same kernel with other sizes of shared memory, which one thread's calls must not take from
    the other's."""
    jobs = []
    for query in (12, 16):
        p = Problem(LENS, 8, nodes=query, query=query, seed=query)
        b = torch.randn((p.num_pages, 8, 2, D), device="cuda").sort(dim=2).values.to(torch.bfloat16)
        outs = [torch.full((len(LENS), query, 8, p.table.shape[1]), 7.0, device="cuda") for _ in range(2)]
        kvshot.page_scores(p.desc, p.q, b, p.t_table, p.t_lens, outs[0])
        jobs.append((p, b, outs, torch.cuda.Stream()))
    torch.cuda.synchronize()
    start, refused = threading.Barrier(len(jobs)), []

    def work(p, b, outs, stream):
        start.wait()
        handle = stream.cuda_stream
        for _ in range(CALLS):
            status = kvshot.page_scores_status(p.desc, p.q, b, p.t_table, p.t_lens, outs[1], handle)
            if status != kvshot.KVSHOT_OK:
                refused.append(status)
    threads = [threading.Thread(target=work, args=job) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not refused, f"{len(refused)} of {CALLS * len(jobs)} calls refused: {refused[0]}"
    for p, _, outs, _ in jobs:
        assert int(p.err.item()) == 0 and torch.equal(*outs)
