"""InertiaKV decode-step eviction path on GB300 (sm_103a): Python side.

``ikv`` binds the C ABI of ``libikv.so`` (include/ikv.h).  ``DecodeCache``
allocates the device tensors a caller hands to that ABI -- paged K/V pools,
block table, lengths, positions, utilities, budgets and workspace -- using
PyTorch purely as the device allocator.  All arithmetic of the path runs in
the CUDA library.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import ikv

__all__ = ["ikv", "DecodeCache", "Q4Cache", "RankTrace", "step_lengths", "auto_max_holes"]


def auto_max_holes(budgets: Sequence[int]) -> int:
    """A deferred-compaction threshold (ikv_params.max_holes) for sequences with these
    budgets.  Holding on average max_holes / 2 dead slots makes the attention read that
    many masked rows per step, and one compaction of about B rows (read + write) is
    spread over max_holes steps; max_holes / 2 + 2 B / max_holes is smallest at
    max_holes = 2 sqrt(B).  Rounded to a multiple of 8, at least 8."""
    import math

    b = sum(budgets) / max(1, len(budgets))
    return max(8, int(round(2 * math.sqrt(b) / 8)) * 8)


def step_lengths(lens: Sequence[int], live: Sequence[int], budgets: Sequence[int], max_holes: int = 0):
    """Host mirror of one ikv_step's length bookkeeping, for sizing max_len.

    lens: slots in use per sequence (len[b], dead slots included); live: live slots.
    The step appends one token; if more than budget[b] slots are then live, it keeps
    budget[b] of them.  The evicted slots are only marked dead while the dead slots
    stay <= max_holes (> 0); otherwise the sequence is compacted to its live slots.
    Returns the (lens, live) after the step."""
    out_l, out_v = [], []
    for L, n, B in zip(lens, live, budgets):
        L, n = L + 1, n + 1
        kept = min(n, B)
        if max_holes > 0 and L - kept <= max_holes:
            out_l.append(L)
        else:
            out_l.append(kept)
        out_v.append(kept)
    return out_l, out_v


class DecodeCache:
    """Device buffers of one batch of decode sequences.

    k, v:        [layers][num_pages][kv_heads][page_size][head_dim] (bf16 or fp32)
    block_table: [batch][max_pages] int32 physical page of each logical page
    len:         [batch] int32 slots in use (dead slots included);  next_pos: [batch] int32
    pos, ema:    [rows][cap] int32 / fp32, rows = batch (per-sequence state) or batch * kv_heads;
                 pos = -1 marks a dead slot (deferred compaction).  With pos_cap > 0 (per-layer
                 eviction): pos has batch * layers rows (row b * layers + l: layer l's positions)
                 and pos_state [batch][pos_cap] is the utility by token position
    budget:      [batch] int32
    With pool_pages, sequences own no page at first: pool_pages pages (numbers 1 ..) are handed out by
    the ikv_pages_* calls, refs [num_pages] counts their holders, block_table entries of 0 mean none, and
    writable [batch][2] names the slots that ikv_pages_writable made each sequence's own.
    """

    def __init__(self, batch: int, layers: int, q_heads: int, kv_heads: int, head_dim: int, cap_tokens: int,
                 dtype: int = ikv.IKV_BF16, page_size: int = 64, granularity: int = ikv.IKV_GRAN_SEQ,
                 device: str = "cuda", page_perm_seed: Optional[int] = None, value_norms: bool = False,
                 pos_cap: int = 0, pool_pages: Optional[int] = None):
        self.batch, self.layers, self.q_heads, self.kv_heads, self.head_dim = batch, layers, q_heads, kv_heads, head_dim
        self.dtype, self.granularity, self.page_size = dtype, granularity, page_size
        self.max_pages = (cap_tokens + page_size - 1) // page_size
        self.cap = self.max_pages * page_size
        self.num_pages = batch * self.max_pages if pool_pages is None else pool_pages + 1
        tdt = torch.bfloat16 if dtype == ikv.IKV_BF16 else torch.float32
        self.torch_dtype = tdt
        self._alloc_pools((layers, self.num_pages, kv_heads, page_size), device)
        # pages handed out as sequences grow (ikv_pages_*): no sequence holds one yet, and page 0
        # stands for none; otherwise every sequence owns max_pages pages for good
        self.refs = self.writable = None
        if pool_pages is not None:
            self.writable = torch.zeros((batch, 2), dtype=torch.int32, device=device)
            self.refs = torch.zeros(self.num_pages, dtype=torch.int32, device=device)
            self.refs[0] = 1
        pages = torch.arange(self.num_pages, dtype=torch.int32)
        if page_perm_seed is not None:
            g = torch.Generator().manual_seed(page_perm_seed)
            pages = pages[torch.randperm(self.num_pages, generator=g)]
        if pool_pages is None:
            self.block_table = pages.view(batch, self.max_pages).to(device)
        else:
            self.block_table = torch.zeros((batch, self.max_pages), dtype=torch.int32, device=device)
        self.rows = batch if granularity == ikv.IKV_GRAN_SEQ else batch * kv_heads
        self.len = torch.zeros(batch, dtype=torch.int32, device=device)
        self.next_pos = torch.zeros(batch, dtype=torch.int32, device=device)
        # per-layer eviction (pos_cap > 0): a position row per (sequence, layer) and the
        # utility state indexed by token position (pos_state); the step-end mode reads
        # the first `rows` position rows and ema
        self.pos_cap = pos_cap
        pos_rows = max(self.rows, batch * layers) if pos_cap > 0 else self.rows
        self.pos = torch.zeros((pos_rows, self.cap), dtype=torch.int32, device=device)
        self.ema = torch.zeros((self.rows, self.cap), dtype=torch.float32, device=device)
        self.pos_state = (torch.zeros((batch, pos_cap), dtype=torch.float32, device=device) if pos_cap > 0
                          else None)
        self.budget = torch.zeros(batch, dtype=torch.int32, device=device)
        self.start = torch.zeros(batch, dtype=torch.int32, device=device)
        # per-slot value-row norms, for the VNorm scorer
        self.vnorm = (torch.zeros((layers, batch, kv_heads, self.cap), dtype=torch.float32, device=device)
                      if value_norms else None)
        self.max_len = 0

    code_bits = 0  # ikv_cache.code_bits: rows of dtype

    def _alloc_pools(self, shp, device) -> None:
        self.k = torch.zeros(shp + (self.head_dim,), dtype=self.torch_dtype, device=device)
        self.v = torch.zeros(shp + (self.head_dim,), dtype=self.torch_dtype, device=device)

    def planes(self):
        """The arrays paged alike, for the ikv_pages_* calls."""
        return [self.k, self.v]

    # ---- ABI structs ------------------------------------------------------
    def pages(self) -> ikv.ikv_pages:
        return ikv.ikv_pages_of(self.refs, self.planes())

    def pages_workspace(self) -> torch.Tensor:
        n = ikv.ikv_pages_workspace_size(self.shape(), self.cache(), self.pages())
        return torch.empty(n, dtype=torch.uint8, device=self.k.device)

    def shape(self) -> ikv.ikv_shape:
        return ikv.ikv_shape(self.batch, self.layers, self.q_heads, self.kv_heads, self.head_dim, self.dtype,
                             self.granularity)

    def cache(self, max_len: Optional[int] = None, dead_slots: bool = False,
              granted: Optional[bool] = None) -> ikv.ikv_cache:
        """granted: stores and appends go by what ikv_pages_writable granted (ikv_cache.writable; steps refuse
        that); the page calls then get it too.  None: a pool of 4-bit rows, which no step serves, does."""
        if granted is None:
            granted = self.code_bits == 4 and self.writable is not None
        ml = self.max_len if max_len is None else max_len
        return ikv.ikv_cache(self.k.data_ptr(), self.v.data_ptr(), self.block_table.data_ptr(), self.num_pages,
                             self.page_size, self.max_pages, self.len.data_ptr(), self.pos.data_ptr(),
                             self.next_pos.data_ptr(), ml, self.start.data_ptr(), 1 if dead_slots else 0,
                             self.vnorm.data_ptr() if self.vnorm is not None else None, self.pos_cap, self.code_bits,
                             self.writable.data_ptr() if granted else None)

    @property
    def rows_per_seq(self) -> int:
        return 1 if self.granularity == ikv.IKV_GRAN_SEQ else self.kv_heads

    # ---- host-side helpers (setup / inspection) ----------------------------
    def set_prefill(self, lengths: Sequence[int], budgets: Sequence[int]) -> None:
        """Mark slots [0, L0_b) as holding positions 0..L0_b-1 with utility 0 (m_0 = 0)."""
        dev = self.len.device
        self.len.copy_(torch.tensor(list(lengths), dtype=torch.int32, device=dev))
        self.next_pos.copy_(self.len)
        self.budget.copy_(torch.tensor(list(budgets), dtype=torch.int32, device=dev))
        ar = torch.arange(self.cap, dtype=torch.int32, device=dev)
        self.pos.copy_(ar.expand(self.pos.shape[0], self.cap))
        self.ema.zero_()
        if self.pos_state is not None:
            self.pos_state.zero_()
        self.start.zero_()
        self.max_len = max(lengths)

    def slot_rows(self, b: int, layer: int, g: int, n: int):
        """(pages, offsets) of cache slots 0..n-1 of sequence b (through start and the block table)."""
        slots = torch.arange(n, device=self.k.device) + int(self.start[b].item())
        pages = self.block_table[b, (slots // self.page_size).long()].long()
        return pages, slots % self.page_size

    def gather(self, pool: torch.Tensor, b: int, layer: int, g: int, n: int) -> torch.Tensor:
        pages, off = self.slot_rows(b, layer, g, n)
        return pool[layer, pages, g, off]

    def scatter(self, pool: torch.Tensor, b: int, layer: int, g: int, rows: torch.Tensor, start: int = 0) -> None:
        n = rows.shape[0]
        s0 = start + int(self.start[b].item())
        slots = torch.arange(s0, s0 + n, device=pool.device)
        pages = self.block_table[b, (slots // self.page_size).long()].long()
        pool[layer, pages, g, slots % self.page_size] = rows.to(pool.dtype)

    def utility(self, evict_mode: int = ikv.IKV_EVICT_STEP) -> torch.Tensor:
        """The utility array a step of this eviction mode updates (ema or pos_state)."""
        return self.pos_state if evict_mode == ikv.IKV_EVICT_LAYER else self.ema

    def step_workspace(self) -> torch.Tensor:
        """Zero-filled, so steps may run with ikv_params.ws_zeroed from the first one."""
        n = ikv.ikv_step_workspace_size(self.shape(), self.cache(self.cap - 1))
        return torch.zeros(n, dtype=torch.uint8, device=self.k.device)

    # ---- attention over a shared prefix, and through a window --------------
    def prefix(self, groups: Sequence[Sequence[int]], lengths: Sequence[int]) -> ikv.ikv_prefix:
        """The groups of ikv_prefix_attend_score: the sequences of each, the one whose pages are read first, and
        the slots they share.  The struct keeps its device tensors (first, member and length_tensor, which may be
        rewritten as the lengths change)."""
        if len(groups) != len(lengths):
            raise ValueError("a length for each group")
        member = [b for g in groups for b in g]
        if len(set(member)) != len(member) or any(not 0 <= b < self.batch for b in member):
            raise ValueError("each sequence belongs to one group at most")
        first = [0]
        for g in groups:
            first.append(first[-1] + len(g))
        t = [torch.tensor(list(x) or [0], dtype=torch.int32, device=self.k.device) for x in (first, member, lengths)]
        p = ikv.ikv_prefix(len(groups), *[x.data_ptr() for x in t])
        p.first_tensor, p.member_tensor, p.length_tensor = t  # (the struct holds their addresses)
        return p

    def prefix_workspace(self, prefix: ikv.ikv_prefix) -> torch.Tensor:
        n = ikv.ikv_prefix_workspace_size(self.shape(), self.cache(), prefix)
        return torch.empty(n, dtype=torch.uint8, device=self.k.device)

    def window(self, window: int, sinks: int, counts: Sequence[int], q_stride: int = 0,
               out_stride: int = 0) -> ikv.ikv_window:
        """What ikv_window_attend is asked for, with the queries of all sequences packed one behind another:
        counts[b] of sequence b.  The struct keeps its device tensors."""
        if len(counts) != self.batch or any(n < 0 for n in counts):
            raise ValueError("a number of queries for each sequence")
        row0 = [sum(counts[:b]) for b in range(self.batch)]
        t = [torch.tensor(x, dtype=torch.int32, device=self.k.device) for x in (row0, list(counts))]
        w = ikv.ikv_window(window, sinks, t[0].data_ptr(), t[1].data_ptr(), max(counts), q_stride, out_stride)
        w.row0_tensor, w.count_tensor = t  # (the struct holds their addresses)
        return w

    def window_workspace(self, window: ikv.ikv_window) -> torch.Tensor:
        n = ikv.ikv_window_workspace_size(self.shape(), self.cache(), window)
        return torch.empty(n, dtype=torch.uint8, device=self.k.device)

    def params(self, alpha: float, refresh_period: int = 1, score_free: bool = False,
               compact_mode: int = ikv.IKV_COMPACT_STABLE, refresh_init: int = ikv.IKV_INIT_ZERO,
               layer_eligible: Optional[Sequence[int]] = None, max_holes: int = 0,
               agg_mode: int = ikv.IKV_AGG_EMA, scorer: int = ikv.IKV_SCORE_ATTENTION,
               evict_mode: int = ikv.IKV_EVICT_STEP, trace: "Optional[RankTrace]" = None,
               ws_zeroed: bool = False) -> ikv.ikv_params:
        p = ikv.ikv_params()
        p.alpha = alpha
        p.refresh_period = refresh_period
        p.score_free = 1 if score_free else 0
        p.budget = self.budget.data_ptr()
        if layer_eligible is not None:
            self._elig = (ctypes_u8 * self.layers)(*[1 if x else 0 for x in layer_eligible])
            p.layer_eligible = ctypes_addr(self._elig)
        p.compact_mode = compact_mode
        p.refresh_init = refresh_init
        p.max_holes = max_holes
        p.agg_mode = agg_mode
        p.scorer = scorer
        p.evict_mode = evict_mode
        p.ws_zeroed = 1 if ws_zeroed else 0
        if trace is not None:
            p.trace = _ct.pointer(trace.struct)
            self._trace = trace
        return p


class Q4Cache(DecodeCache):
    """A DecodeCache held in 4 bits (include/ikv.h, "Caches held in 4 bits"): k and v are code pools
    [layers][num_pages][kv_heads][page_size][head_dim / 2], k_scale and v_scale their scales; dtype is
    the type of q, out and of the rows that ikv_q4_store takes.  The calls for dense rows refuse it; to
    evict from it, give it pool_pages (ikv_pages_compact)."""

    code_bits = 4

    def _alloc_pools(self, shp, device) -> None:
        self.k = torch.zeros(shp + (self.head_dim // 2,), dtype=torch.uint8, device=device)
        self.v = torch.zeros(shp + (self.head_dim // 2,), dtype=torch.uint8, device=device)
        self.k_scale = torch.zeros(shp + (self.head_dim // 32,), dtype=torch.bfloat16, device=device)
        self.v_scale = torch.zeros(shp + (self.head_dim // 32,), dtype=torch.bfloat16, device=device)

    def planes(self):
        return [self.k, self.v, self.k_scale, self.v_scale]

    def q4(self) -> ikv.ikv_q4:
        return ikv.ikv_q4(self.k_scale.data_ptr(), self.v_scale.data_ptr())

    def dense_rows(self, k: torch.Tensor, row0: Optional[torch.Tensor] = None) -> ikv.ikv_rows:
        """How dense rows lie: [layers][batch][tokens][kv_heads][head_dim], or packed
        [layers][tokens][kv_heads][head_dim] with the first row of every sequence in row0; any
        strides but the last."""
        st = k.stride()
        if st[-1] != 1:
            raise ValueError("the channels of a row must be contiguous")
        if row0 is not None:
            if row0.dtype != torch.int32 or row0.numel() < self.batch or not row0.is_contiguous():
                raise ValueError("row0 must be contiguous int32, a number for each sequence")
            rows = ikv.ikv_rows(st[0], 0, st[1], st[2], row0.data_ptr())
            rows.row0_tensor = row0  # (the struct holds its address)
            return rows
        return ikv.ikv_rows(st[0], st[1], st[2], st[3], None)

    def attend_workspace(self) -> torch.Tensor:
        n = ikv.ikv_attend_workspace_size(self.shape(), self.cache())
        return torch.empty(n, dtype=torch.uint8, device=self.k.device)


import ctypes as _ct  # noqa: E402

ctypes_u8 = _ct.c_uint8


def ctypes_addr(x) -> int:
    return _ct.addressof(x)


class RankTrace:
    """Device buffers of the rank-trace diagnostics (ikv_trace) for one DecodeCache: each
    utility row's previous raw / EMA top-k positions, their sizes and the last step's
    overlap counts {|R & R_prev|, |E & E_prev|, |R & E|, |R|, |E|}."""

    def __init__(self, c: DecodeCache):
        dev = c.k.device
        self.raw_top = torch.zeros((c.rows, c.cap), dtype=torch.int32, device=dev)
        self.ema_top = torch.zeros((c.rows, c.cap), dtype=torch.int32, device=dev)
        self.n_top = torch.zeros((c.rows, 2), dtype=torch.int32, device=dev)
        self.counts = torch.zeros((c.rows, 5), dtype=torch.int32, device=dev)
        self.struct = ikv.ikv_trace(self.raw_top.data_ptr(), self.ema_top.data_ptr(), self.n_top.data_ptr(),
                                    self.counts.data_ptr())

    def reset(self) -> None:
        self.n_top.zero_()
