"""A 4-bit target cache with its page tables: the state that a drafting server keeps between verification steps.

Between two drafting steps the target has verified some tokens of each sequence.  grow() finds room for them
(kvshot_cache_extend) and quantises their K and V into it (kvshot_kv4_store); DraftStep(target_kv4=...) then drafts over
the cache (kvshot_draft_attn_kv4), and values() reads tokens back (kvshot_kv4_load).  Lengths, tables and the list of
free pages live on the device and are changed there in stream order: a step needs no word from the host, and grow() can
be captured in a graph together with the step (its sizes are those of the buffers it is given).
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import kvshot


class Kv4Cache:
    def __init__(self, num_caches: int, hkv: int, num_pages: int, max_pages_per_seq: int, *, page_size: int = 16,
                 max_tokens: int, k_scale_exp: int = 0, v_scale_exp: int = 0, device="cuda"):
        """max_tokens: the most tokens that one grow() adds, over all caches."""
        size = kvshot.kv4_cache_bytes(num_pages, hkv, page_size)
        if size == 0:
            raise kvshot.KvshotError(kvshot.KVSHOT_ERR_SHAPE, "kvshot_kv4_cache_bytes")
        self.num_caches, self.hkv, self.page_size, self.num_pages = num_caches, hkv, page_size, num_pages
        self.max_pages_per_seq = max_pages_per_seq
        self.k_scale_exp, self.v_scale_exp, self.max_tokens = k_scale_exp, v_scale_exp, max_tokens
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        # Sizes that every call would refuse: without pointers, or tokens, the calls check them and do nothing.
        self._extend = self._extend_desc(max_tokens)
        status = kvshot.cache_extend_status(self._extend, *[None] * 12, stream=0)
        if status != kvshot.KVSHOT_ERR_NULL:
            raise kvshot.KvshotError(status, "kvshot_cache_extend")
        kvshot.kv4_store(self._rows(0), None, None, None, None, stream=0)

        def i32(*shape):
            return torch.zeros(shape, dtype=torch.int32, device=device)

        self.data = torch.empty(size, dtype=torch.uint8, device=device)
        self.seq_lens, self.page_table = i32(num_caches), i32(num_caches, max_pages_per_seq)
        self.free_pages = torch.arange(num_pages - 1, -1, -1, dtype=torch.int32, device=device)  # taken from its end
        self.free_count = torch.full((1,), num_pages, dtype=torch.int32, device=device)
        # Of the last grow(): first packed token of each cache; slot, cache and position of each packed token (or -1).
        self.token_start = i32(num_caches + 1)
        self._maps = i32(3, max_tokens)
        self.slots, self.token_cache, self.positions = self._maps.unbind()

    @property
    def max_seq_len(self) -> int:
        return self.max_pages_per_seq * self.page_size

    def _extend_desc(self, max_tokens: int) -> kvshot.ExtendDesc:
        return kvshot.make_extend_desc(num_caches=self.num_caches, page_size=self.page_size,
                                       max_pages_per_seq=self.max_pages_per_seq, num_pages=self.num_pages,
                                       max_tokens=max_tokens, err_flag=self.err)

    def _rows(self, num_tokens: int, k_stride: int = 0, v_stride: int = 0) -> kvshot.Kv4Desc:
        return kvshot.make_kv4_desc(num_tokens=num_tokens, hkv=self.hkv, page_size=self.page_size,
                                    num_pages=self.num_pages, k_scale_exp=self.k_scale_exp,
                                    v_scale_exp=self.v_scale_exp, k_stride=k_stride, v_stride=v_stride,
                                    err_flag=self.err)

    def extend(self, new_tokens: torch.Tensor, stream=None) -> None:
        """Pages and slots for new_tokens[c] (int32 [num_caches]) more tokens of each cache; self.slots are theirs."""
        self._extend_by(self._extend, new_tokens, stream)

    def _check_ints(self, name: str, x: torch.Tensor, shape=None) -> None:
        """The calls take bare pointers: a tensor of another type or order would be read as other numbers."""
        if x.dtype != torch.int32 or x.device != self.data.device or not x.is_contiguous() or x.dim() != 1 or \
                (shape is not None and x.shape != shape):
            size = "" if shape is None else str(shape[0])
            raise ValueError(f"{name} must be int32 [{size}] on {self.data.device}, and contiguous")

    def _extend_by(self, desc: kvshot.ExtendDesc, new_tokens: torch.Tensor, stream) -> None:
        self._check_ints("new_tokens", new_tokens, (self.num_caches,))
        kvshot.cache_extend(desc, self.seq_lens, new_tokens, self.page_table, self.free_pages, self.free_count,
                            self.seq_lens, self.page_table, self.free_count, self.token_start, self.slots,
                            self.token_cache, self.positions, stream)

    def _store_desc(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> kvshot.Kv4Desc:
        """The descriptor of a store, with everything checked that would make the call refuse it or misread its rows."""
        t = k.shape[0] if k.dim() == 3 else 0
        if k.shape != v.shape or k.shape[1:] != (self.hkv, 128) or k.dtype != torch.bfloat16 or v.dtype != torch.bfloat16:
            raise ValueError(f"k and v must be bf16 [T, {self.hkv}, 128]")
        if t > slots.shape[0]:
            raise ValueError(f"{t} tokens for {slots.shape[0]} slots")
        for x in (k, v):
            if x.device != self.data.device:
                raise ValueError(f"k and v must be on {self.data.device}")
            if t == 0:
                continue
            if x.stride()[1:] != (128, 1) or x.data_ptr() % 16:
                raise ValueError("a token's heads must be contiguous, from 16-byte aligned addresses on")
            if t > 1 and (x.stride(0) < self.hkv * 128 or x.stride(0) % 8):
                raise ValueError("tokens must lie apart by a multiple of 8 elements, and not over one another")
        return self._rows(t, *((k.stride(0), v.stride(0)) if t > 1 else (0, 0)))

    def store(self, k: torch.Tensor, v: torch.Tensor, slots: Optional[torch.Tensor] = None, stream=None) -> None:
        """K and V [T, hkv, 128] (bf16; rows may be slices of wider ones) into slots [T] (default: the first T of
        self.slots)."""
        slots = self.slots if slots is None else slots
        self._check_ints("slots", slots)
        desc = self._store_desc(k, v, slots)
        if desc.num_tokens:
            kvshot.kv4_store(desc, k, v, slots, self.data, stream)

    def grow(self, new_tokens: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """extend(), then store(): K and V packed cache after cache.  Rows past the new tokens are not stored.  Nothing is
        enqueued if K or V are refused, and nothing taken if the rows are fewer than the new tokens (which the device
        finds, as extend() its other errors)."""
        desc, t = self._store_desc(k, v, self.slots), k.shape[0]
        self._extend_by(self._extend_desc(t), new_tokens, stream)
        if t < self.max_tokens:  # (the maps of an extension by t tokens at most end there)
            with kvshot.torch_stream(stream):
                self._maps[:, t:].fill_(-1)
        if t:
            kvshot.kv4_store(desc, k, v, self.slots, self.data, stream)

    def values(self, slots: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """K and V [T, hkv, 128] (bf16) of slots [T]; -1 gives zeros.  Both are memory of `stream`, like its own tensors."""
        self._check_ints("slots", slots)
        shape = (slots.shape[0], self.hkv, 128)
        with kvshot.torch_stream(stream):
            k, v = (torch.empty(shape, dtype=torch.bfloat16, device=self.data.device) for _ in range(2))
        if slots.shape[0]:
            kvshot.kv4_load(self._rows(slots.shape[0]), self.data, slots, k, v, stream)
        return k, v

    def error_code(self) -> int:
        """The first error that the cache's calls have recorded since the last time this was asked (0: none)."""
        code = int(self.err.item())
        if code:
            self.err.zero_()
        return code


def of_inputs(inp, page_size: int = 16, spare_pages: int = 0, spare_tokens: int = 0, k_exp: int = 0,
              v_exp: int = 0) -> Kv4Cache:
    """A 4-bit cache that holds the target prefixes of inp (workloads.Inputs), stored through the library, with spare_pages
    more pages in the pool and room for spare_tokens more tokens of each cache."""
    s, lens = inp.spec, inp.seq_lens
    pages = [-(-n // page_size) for n in s.seq_lens]
    row = max(1, -(-(s.max_seq_len + spare_tokens) // page_size))
    cache = Kv4Cache(s.num_caches, s.hkv, max(1, sum(pages) + spare_pages), row, page_size=page_size,
                     max_tokens=max(1, sum(s.seq_lens), spare_tokens * s.num_caches), k_scale_exp=k_exp,
                     v_scale_exp=v_exp, device=inp.target_k.device)
    cache.extend(lens)
    n = sum(s.seq_lens)
    c, pos = cache.token_cache[:n].long(), cache.positions[:n].long()
    size = s.page_size if inp.page_table is not None else inp.l_cap
    page = inp.page_table[c, pos // size].long() if inp.page_table is not None else c
    cache.store(inp.target_k[page, :, pos % size], inp.target_v[page, :, pos % size])
    return cache
