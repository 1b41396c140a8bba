"""One drafting step of the hot path through the C ABI.

A step drafts every level of the draft chain/tree once: for each drafting
step d (Nq_d new nodes), the new nodes' q/k/v are RoPE'd and appended
(kvshot_draft_append), then the new nodes attend over [target prefix | draft
KV so far] (kvshot_draft_attn).  In "whole" mode all N nodes are appended
once and attend together (whole-tree verification shape).  The target prefix is
bf16, fp8 or 4 bits; the 4-bit cache grows between steps (kv4.Kv4Cache).  Over a paged bf16 prefix a step may read the best
pages of each node alone, and add up the tokens' softmax weights (partial.PageSelection, partial.TokenWeights).

Only device memory is handled here (torch allocations); all arithmetic runs
in libkvshot's kernels, but for one sum: over a 4-bit cache a step first adds
the cache's present lengths to the nodes' places behind the prefix.
"""
from __future__ import annotations

from typing import List, Optional

import torch

from . import kvshot
from . import workloads as wl
from .kv4 import Kv4Cache
from .partial import PageSelection, TokenWeights


class DraftStep:
    def __init__(self, inp: wl.Inputs, mode: str = "per_depth", flags: int = 0, num_ctas: int = 0,
                 scale: float = 0.0, err_flag: bool = True, target_fp8=None, qk_norm=None,
                 target_kv4: Optional[Kv4Cache] = None, window: int = 0, sinks: int = 0,
                 pages: Optional[PageSelection] = None, weights: Optional[TokenWeights] = None):
        """target_fp8: optional (codes_k, codes_v, k_scale_exp, v_scale_exp), an e4m3 copy of the target
        cache (workloads.fp8_target) to attend instead of inp.target_k / inp.target_v.
        qk_norm: optional (q_norm_w, k_norm_w, eps): the append normalises q and k per head first
        (kvshot_draft_append_qknorm).
        target_kv4: optional 4-bit cache to attend, with its own lengths and tables, instead of inp's target cache;
        then also window and sinks (kvshot_draft_attn_kv4).  Its draft tokens stand behind the lengths that the cache has
        when run() comes to them in stream order: inp's positions only say how far behind inp's lengths a node stands.
        pages: optional selection of inp's pages: each node reads the best ones for it, per KV head.
        weights: optional weights of inp's tokens, to which every level adds (not with pages: a softmax over some tokens gives no
        weights to the others)."""
        if mode not in ("per_depth", "whole"):
            raise ValueError(mode)
        if target_kv4 is None and (window or sinks):
            raise ValueError("a window needs the 4-bit target cache")
        if target_kv4 is not None and target_fp8 is not None:
            raise ValueError("one target cache")
        if (pages is not None or weights is not None) and (target_fp8 is not None or target_kv4 is not None):
            raise ValueError("pages and weights are of the bf16 target cache")
        if pages is not None and weights is not None:
            raise ValueError("weights need the softmax over all tokens")
        if any(x is not None and x.inp is not inp for x in (pages, weights)):
            raise ValueError("pages and weights of another cache")
        self.inp, self.mode = inp, mode
        self.pages, self.weights = pages, weights
        self.qk_norm = qk_norm
        self.kv4, self.window, self.sinks = target_kv4, window, sinks
        s = inp.spec
        k_exp = v_exp = 0
        if target_fp8 is not None:
            self.target_k, self.target_v, k_exp, v_exp = target_fp8
            flags |= kvshot.KVSHOT_TARGET_FP8
        else:
            self.target_k, self.target_v = inp.target_k, inp.target_v
        if target_kv4 is not None:
            if (target_kv4.num_caches, target_kv4.hkv) != (s.num_caches, s.hkv):
                raise ValueError("the 4-bit cache is of other caches or heads")
            k_exp, v_exp = target_kv4.k_scale_exp, target_kv4.v_scale_exp
        dev = inp.target_k.device
        self.device = dev
        C, N = s.num_caches, s.n_nodes
        self.draft_k = torch.zeros((C, s.hkv, inp.n_max, s.head_dim), dtype=torch.bfloat16, device=dev)
        self.draft_v = torch.zeros_like(self.draft_k)
        self.err = torch.zeros(1, dtype=torch.int32, device=dev) if err_flag else None
        if mode == "per_depth":
            self.levels = list(s.levels)
            self.q_in, self.k_in, self.v_in, self.pos = inp.q_in, inp.k_in, inp.v_in, inp.positions
        else:
            self.levels = [N]
            self.q_in = [torch.cat(inp.q_in, dim=1)]
            self.k_in = [torch.cat(inp.k_in, dim=1)]
            self.v_in = [torch.cat(inp.v_in, dim=1)]
            self.pos = [torch.cat(inp.positions, dim=1).contiguous()]
        if target_kv4 is not None:
            self._places_behind_the_cache()
        self.q_rot: List[torch.Tensor] = [torch.empty_like(q) for q in self.q_in]
        self.out: List[torch.Tensor] = [torch.empty_like(q) for q in self.q_in]
        self.lse: List[torch.Tensor] = [torch.empty(q.shape[:3], dtype=torch.float32, device=dev) for q in self.q_in]
        paged = inp.page_table is not None
        cache = dict(max_seq_len=s.max_seq_len, page_size=s.page_size if paged else 0,
                     max_pages_per_seq=inp.page_table.shape[1] if paged else 0,
                     num_pages=inp.num_pages if paged else 0, l_cap=inp.l_cap)
        if target_kv4 is not None:
            cache = dict(max_seq_len=target_kv4.max_seq_len, page_size=target_kv4.page_size,
                         max_pages_per_seq=target_kv4.page_table.shape[1], num_pages=target_kv4.num_pages)
        self.descs = []
        self.parents: List[torch.Tensor] = []  # [B, n_nodes] of each call (tree_parent's row stride is n_nodes)
        n0 = 0
        for n_step in self.levels:
            n0 += n_step
            self.parents.append(inp.tree_parent[:, :n0].contiguous())
            self.descs.append(kvshot.make_desc(
                num_caches=C, num_seqs=s.num_seqs, hq=s.hq, hkv=s.hkv, n_nodes=n0, n_query=n_step,
                n_max=inp.n_max, head_dim=s.head_dim, scale=scale, tree=s.tree, **cache,
                # the attention call follows this step's own append kernel, which writes only q and the draft K/V
                flags=flags | kvshot.KVSHOT_OVERLAP_PREVIOUS, num_ctas=num_ctas, err_flag=self.err,
                k_scale_exp=k_exp, v_scale_exp=v_exp))
        if target_kv4 is not None:
            ws = [kvshot.draft_attn_kv4_workspace_size(d, window, sinks) for d in self.descs]
        elif pages is not None:
            ws = [kvshot.draft_attn_sparse_workspace_size(d, pages.keep) for d in self.descs]
            self._pick_buffers()
        else:
            ws = [kvshot.workspace_size(d) for d in self.descs]
        ws = max(ws) if min(ws) > 0 else 0
        if ws == 0:
            raise kvshot.KvshotError(kvshot.KVSHOT_ERR_SHAPE, "kvshot_draft_attn_workspace_size")
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=dev)
        for d in self.descs:
            d.workspace = self.workspace.data_ptr()
            d.workspace_bytes = ws

    def _pick_buffers(self) -> None:
        """Of every level: scores of the pages, the picks and their numbers."""
        s, dev, width = self.inp.spec, self.device, self.inp.page_table.shape[1]
        self.select = [self.pages.select_desc(n) for n in self.levels]
        rows = [(s.num_caches, n, s.hkv) for n in self.levels]
        self.scores = [torch.empty((*r, width), dtype=torch.float32, device=dev) for r in rows]
        self.picks = [torch.empty((*r, self.pages.keep), dtype=torch.int32, device=dev) for r in rows]
        self.counts = [torch.empty(r, dtype=torch.int32, device=dev) for r in rows]

    @property
    def tokens(self) -> int:
        """Draft tokens produced per step (a token attending several reused layers counts once)."""
        return self.inp.spec.num_seqs * self.inp.spec.n_nodes

    def _places_behind_the_cache(self) -> None:
        """Positions of the step's own, and the sums that fill them: consecutive levels of one width take one launch."""
        behind = [p - self.inp.seq_lens[:, None] for p in self.pos]
        C, self.pos, self._sums, i = len(self.inp.seq_lens), [], [], 0
        while i < len(behind):
            j, n = i, behind[i].shape[1]
            while j < len(behind) and behind[j].shape[1] == n:
                j += 1
            place = torch.empty((j - i, C, n), dtype=torch.int32, device=self.device)
            self._sums.append((torch.stack(behind[i:j]), place))
            self.pos += list(place.unbind())
            i = j

    def run(self, stream: Optional[torch.cuda.Stream] = None) -> None:
        inp = self.inp
        if self.kv4 is not None:
            with kvshot.torch_stream(stream):
                for behind, place in self._sums:
                    torch.add(behind, self.kv4.seq_lens[:, None], out=place)
        stream = kvshot._stream(stream)  # once for all calls
        n0 = 0
        for i, n_step in enumerate(self.levels):
            d = self.descs[i]
            if self.qk_norm is not None:
                wq, wk, eps = self.qk_norm
                kvshot.draft_append_qknorm(d, self.q_in[i], self.k_in[i], self.v_in[i], self.pos[i], n0, n_step,
                                           inp.spec.rope_base, wq, wk, eps, self.draft_k, self.draft_v,
                                           self.q_rot[i], stream)
            else:
                kvshot.draft_append(d, self.q_in[i], self.k_in[i], self.v_in[i], self.pos[i], n0, n_step,
                                    inp.spec.rope_base, self.draft_k, self.draft_v, self.q_rot[i], stream)
            if self.kv4 is not None:
                kvshot.draft_attn_kv4(d, self.q_rot[i], self.kv4.data, self.kv4.page_table, self.kv4.seq_lens,
                                      self.draft_k, self.draft_v, self.parents[i], self.window, self.sinks,
                                      self.out[i], self.lse[i], stream)
            elif self.pages is not None:
                kvshot.page_scores(d, self.q_rot[i], self.pages.bounds, inp.page_table, inp.seq_lens, self.scores[i], stream)
                kvshot.select_top(self.select[i], self.scores[i], inp.seq_lens, self.picks[i], self.counts[i], stream)
                kvshot.draft_attn_sparse(d, self.q_rot[i], inp.target_k, inp.target_v, inp.page_table, inp.seq_lens,
                                         self.picks[i], self.counts[i], self.pages.keep, self.draft_k, self.draft_v,
                                         self.parents[i], self.out[i], self.lse[i], stream)
            else:
                kvshot.draft_attn(d, self.q_rot[i], self.target_k, self.target_v, inp.page_table, inp.seq_lens,
                                  self.draft_k, self.draft_v, self.parents[i], self.out[i], self.lse[i], stream)
            if self.weights is not None:
                self.weights.add(d, self.q_rot[i], self.lse[i], stream)
            n0 += n_step

    def error_code(self) -> int:
        """An error that the step's calls have recorded, or else its selection's (PageSelection.error_code ends that one); 0:
        none."""
        code = int(self.err.item()) if self.err is not None else 0
        return code or (int(self.pages.err.item()) if self.pages is not None else 0)
