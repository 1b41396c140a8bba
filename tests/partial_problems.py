"""Small problems for the entry points that draft over a part of a long cache: device tensors and their fp64 copies."""
from __future__ import annotations

import numpy as np
import torch

from paper_2604_26412_gb300 import kvshot

D = 128


def f64(x):
    return x.float().cpu().numpy().astype(np.float64)


class Problem:
    """Caches of given lengths in a shuffled pool with spare pages, every token past a length NaN, and query rows."""

    def __init__(self, lens, page, hq=32, hkv=8, nodes=1, query=1, tree=False, layers=1, seed=0, contiguous=False,
                 scale=0.0, std=0.5, device="cuda"):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.lens, self.page, self.hq, self.hkv, self.N, self.Nq, self.layers = np.asarray(lens), page, hq, hkv, nodes, query, layers
        self.scale = scale or 1 / np.sqrt(D)
        c = len(lens)
        used = -(-self.lens // page)
        width = max(1, int(used.max())) + 1
        self.num_pages = int(used.sum()) + 5
        ids = rng.permutation(self.num_pages)
        self.table = np.full((c, width), -7, np.int32)  # (entries past a cache's last page are nobody's to read)
        self.table[np.arange(width)[None] < used[:, None]] = ids[:int(used.sum())]
        self.free = ids[int(used.sum()):].astype(np.int32)
        l_cap = max(1, int(self.lens.max())) + 3
        shape = (c, hkv, l_cap, D) if contiguous else (self.num_pages, hkv, page, D)

        def randn(*s, scale=1.0):
            return (torch.randn(s, generator=g) * scale).to(torch.bfloat16)
        k, v = randn(*shape), randn(*shape)
        live = torch.zeros(shape[0], shape[2], dtype=torch.bool)
        for i, n in enumerate(self.lens):
            if contiguous:
                live[i, :n] = True
            else:
                for p in range(int(used[i])):
                    live[self.table[i, p], :min(page, int(n) - p * page)] = True
        for x in (k, v):
            x.masked_fill_(~live[:, None, :, None], float("nan"))
        slots = nodes + 3
        dk, dv = randn(c, hkv, slots, D), randn(c, hkv, slots, D)
        dk[:, :, nodes:], dv[:, :, nodes:] = float("nan"), float("nan")
        self.parent = None
        if tree:
            self.parent = np.stack([[int(rng.integers(-1, i)) if i else -1 for i in range(nodes)]
                                    for _ in range(c // layers)]).astype(np.int32)
        self.q, self.k, self.v, self.dk, self.dv = (x.to(device) for x in (randn(c, query, hq, D, scale=std / 0.1), k, v, dk, dv))
        self.q *= 0.1
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        self.t_lens, self.t_table = self.ints(self.lens), None if contiguous else self.ints(self.table)
        self.t_parent = None if self.parent is None else self.ints(self.parent)
        self.desc = kvshot.make_desc(
            num_caches=c, num_seqs=c // layers, hq=hq, hkv=hkv, n_nodes=nodes, n_query=query, n_max=slots,
            max_seq_len=max(int(self.lens.max()), 1), page_size=0 if contiguous else page,
            max_pages_per_seq=0 if contiguous else width, num_pages=0 if contiguous else self.num_pages,
            l_cap=l_cap if contiguous else 0, tree=tree, scale=scale, err_flag=self.err)

    def ints(self, x):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(self.err.device if hasattr(self, "err") else "cuda")

    def random_picks(self, keep, seed=0):
        """Ascending page lists of every (cache, row, KV head), of lengths from 0 to keep."""
        rng = np.random.default_rng(seed)
        c = len(self.lens)
        picks, counts = np.full((c, self.Nq, self.hkv, keep), -1, np.int32), np.zeros((c, self.Nq, self.hkv), np.int32)
        for i in range(c):
            pages = -(-int(self.lens[i]) // self.page)
            for n in range(self.Nq):
                for h in range(self.hkv):
                    m = int(rng.integers(0, min(pages, keep) + 1)) if (i + n + h) % 3 else min(pages, keep)
                    picks[i, n, h, :m] = np.sort(rng.permutation(pages)[:m])
                    counts[i, n, h] = m
        return picks, counts

    def workspace(self, keep):
        size = kvshot.draft_attn_sparse_workspace_size(self.desc, keep)
        assert size > 0
        ws = torch.full((size,), 0xA5, dtype=torch.uint8, device=self.err.device)
        self.desc.workspace, self.desc.workspace_bytes = ws.data_ptr(), size
        return ws
