"""Drafting over a part of a long target cache: which pages a draft token reads, and which tokens a cache keeps.

PageSelection holds the bounds of the pages' keys (kvshot_page_bounds); update() brings them up to date after the cache
grew.  DraftStep(pages=...) scores every page for every draft token and KV head (kvshot_page_scores), picks the best
(kvshot_select_top) and attends to those and the draft K/V (kvshot_draft_attn_sparse).

TokenWeights adds up the softmax weight that each cached token gets (kvshot_key_weights); DraftStep(weights=...) adds to it
at every level.  evict() keeps the tokens with the most (kvshot_select_top), moves them to the front of their cache and gives
the other pages back (kvshot_cache_evict); the bounds of every PageSelection of that cache follow.

Both are of a paged bf16 cache, as workloads.Inputs holds one.  All of it is enqueued on the device in stream order, with
sizes known beforehand, and can be captured in a graph together with the step.
"""
from __future__ import annotations

import weakref
from typing import Optional

import torch

from . import kvshot


def _paged(inp) -> None:
    if inp.page_table is None:
        raise ValueError("a paged target cache is needed")


def _selections(inp) -> weakref.WeakSet:
    """The PageSelections of inp's pages, whose bounds have to follow when its keys move."""
    return vars(inp).setdefault("selections", weakref.WeakSet())


def _reported(err) -> int:
    code = int(err.item())
    if code:
        err.zero_()
    return code


def _check_select(**sizes) -> kvshot.SelectDesc:
    """A descriptor whose sizes the call does not refuse (without pointers it checks them and does nothing)."""
    desc = kvshot.make_select_desc(**sizes)
    status = kvshot.select_top_status(desc, None, None, None, None, stream=0)
    if status not in (kvshot.KVSHOT_OK, kvshot.KVSHOT_ERR_NULL):
        raise kvshot.KvshotError(status, "kvshot_select_top")
    return desc


class PageSelection:
    def __init__(self, inp, keep: int, first: int = 1, last: int = 4):
        """keep: pages that a draft token reads for each KV head, the cache's first `first` and last `last` ones among them."""
        _paged(inp)
        s = inp.spec
        self.inp, self.keep, self.first, self.last = inp, keep, first, last
        self.err = torch.zeros(1, dtype=torch.int32, device=inp.target_k.device)
        self._desc = kvshot.make_desc(num_caches=s.num_caches, num_seqs=s.num_seqs, hq=s.hq, hkv=s.hkv, n_nodes=0, n_query=0,
                                      n_max=0, head_dim=s.head_dim, max_seq_len=inp.page_table.shape[1] * s.page_size,
                                      page_size=s.page_size, max_pages_per_seq=inp.page_table.shape[1],
                                      num_pages=inp.num_pages, err_flag=self.err)
        self.select_desc(1)
        self.bounds = torch.empty((inp.num_pages, s.hkv, 2, s.head_dim), dtype=torch.bfloat16, device=inp.target_k.device)
        self.update()
        _selections(inp).add(self)

    def update(self, from_tokens: Optional[torch.Tensor] = None, stream=None) -> None:
        """Bounds of the pages that hold tokens at or past from_tokens (int32 [num_caches], lengths before the cache grew;
        default: of all pages)."""
        inp = self.inp
        if from_tokens is not None and (from_tokens.dtype != torch.int32 or from_tokens.shape != inp.seq_lens.shape
                                        or not from_tokens.is_contiguous() or from_tokens.device != inp.seq_lens.device):
            raise ValueError(f"from_tokens must be int32 [{inp.seq_lens.shape[0]}] on {inp.seq_lens.device}, and contiguous")
        kvshot.page_bounds(self._desc, inp.target_k, inp.page_table, inp.seq_lens, from_tokens, self.bounds, stream)

    def select_desc(self, n_query: int) -> kvshot.SelectDesc:
        s, pages = self.inp.spec, self.inp.page_table.shape[1]
        return _check_select(num_rows=s.num_caches * n_query * s.hkv, row_len=pages, rows_per_len=n_query * s.hkv,
                             tokens_per_entry=s.page_size, keep=self.keep, first=self.first, last=self.last,
                             err_flag=self.err)

    def error_code(self) -> int:
        """The first error that the bounds' and the selection's calls have recorded since the last time this was asked (0:
        none)."""
        return _reported(self.err)


class TokenWeights:
    def __init__(self, inp, decay: float = 1.0):
        """decay: what is left of a token's weight when a level's is added."""
        _paged(inp)
        s, dev = inp.spec, inp.target_k.device
        self.inp, self.decay = inp, decay
        self.width = inp.page_table.shape[1] * s.page_size
        self.weights = torch.zeros((s.num_caches, self.width), dtype=torch.float32, device=dev)
        self.err = torch.zeros(1, dtype=torch.int32, device=dev)
        # The pages that eviction gives back: entries of the list that kvshot_cache_extend takes from.
        self.free_pages = torch.full((inp.num_pages,), -1, dtype=torch.int32, device=dev)
        self.free_count = torch.zeros(1, dtype=torch.int32, device=dev)
        self._kept = {}
        self._captured = set()

    def add(self, desc: kvshot.AttnDesc, q, lse, stream=None) -> None:
        """The weights of a level's query rows: q and lse as the draft attention took and gave them."""
        inp = self.inp
        kvshot.key_weights(desc, q, inp.target_k, inp.page_table, inp.seq_lens, lse, self.decay, self.width, self.weights,
                           self.weights, stream)

    def evict(self, keep: int, first: int = 4, last: int = 64, stream=None) -> None:
        """Keep `keep` tokens of each cache (all of a shorter one): the first `first`, the last `last`, and the others with the
        most weight.  Changes the cache, its lengths and weights in place, then computes anew the bounds of the selections that
        there are of inp's pages, whose keys are others now.  (Those that are made after an eviction was captured are not in its
        graph: update() them behind it.)"""
        inp, s = self.inp, self.inp.spec
        sizes = (keep, first, last)
        if sizes not in self._kept:  # (buffers of a captured eviction stay as they are)
            select = _check_select(num_rows=s.num_caches, row_len=self.width, keep=keep, first=first, last=last,
                                   err_flag=self.err)
            evict = kvshot.make_evict_desc(num_caches=s.num_caches, hkv=s.hkv, page_size=s.page_size,
                                           max_pages_per_seq=inp.page_table.shape[1], num_pages=inp.num_pages, max_kept=keep,
                                           weights_len=self.width, head_dim=s.head_dim, err_flag=self.err)
            with kvshot.torch_stream(stream):
                self._kept[sizes] = (select, evict, torch.empty((s.num_caches, keep), dtype=torch.int32, device=self.err.device),
                                     torch.empty(s.num_caches, dtype=torch.int32, device=self.err.device))
        select, evict, kept, counts = self._kept[sizes]
        kvshot.select_top(select, self.weights, inp.seq_lens, kept, counts, stream)
        kvshot.cache_evict(evict, inp.target_k, inp.target_v, inp.page_table, inp.seq_lens, kept, counts, self.weights,
                           inp.target_k, inp.target_v, inp.page_table, inp.seq_lens, self.weights, self.free_pages,
                           self.free_count, self.free_count, stream)
        selections = list(_selections(inp))
        if selections:
            with kvshot.torch_stream(stream):
                if torch.cuda.is_current_stream_capturing():
                    self._captured.update(selections)  # (the graph writes their bounds as long as it is replayed)
            for pages in selections:
                pages.update(stream=stream)

    def error_code(self) -> int:
        """The first error that the calls have recorded since the last time this was asked (0: none)."""
        return _reported(self.err)
