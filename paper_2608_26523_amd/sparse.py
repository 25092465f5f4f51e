"""Attention to selected blocks of a paged cache: the torch-facing wrapper of include/vpp_block_attn.h.

``BlockSparseAttention`` stands beside ``ChunkAttention`` where the cost of a chunk must not
grow with its prefix: the cached keys are cut into blocks, each complete block has a summary,
and each query block (one token or a few consecutive ones) attends to the blocks that score
best for it, next to the first and the last ones. The arithmetic runs in the HIP library; there is no other
implementation to fall back to.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as B
from .attention import ChunkAttention
from .rotary import new_on


class BlockSparseAttention:
    """Block-sparse causal attention for one layer's head configuration, chunk by chunk or token by
    token (the chunk's K/V already written to the paged cache)::

        attn = BlockSparseAttention(hq, hkv, dqk, dv, max_blocks=32)
        summaries = attn.new_summaries(num_pages, page_size)        # one per layer, kept with its cache
        attn.plan(cu_q, kv_start, prefix_len)                       # once a chunk
        done = attn.completed(cu_q, kv_start, prefix_len, host_table, page_size)
        attn.summarize(k_pages, done, summaries)                    # these three every layer
        blocks = attn.select(q, summaries, block_table)
        out, lse = attn.run_paged(q, k_pages, v_pages, block_table, blocks)

    ``block_size`` keys a block (64, 128 or 256, at most a page); ``query_block`` tokens share a list
    of ``max_blocks`` blocks, of which the request's first ``sink_blocks``, the ``local_blocks`` up to
    that of the query block's first token and those of its own tokens are always part.

    A plan's query blocks are on the device, copied there on the stream that is current at
    ``plan``; runs on another stream wait for that copy. A run that is captured into a graph reads
    the plan it was captured under: plan before the capture, keep this object, and do not plan it
    again while such a graph is replayed. Workspaces are allocated by each call (within a capture
    from the graph's own memory), so calls on several streams share none.
    """

    def __init__(self, num_q_heads: int, num_kv_heads: int, head_dim_qk: int, head_dim_v: int, max_blocks: int,
                 block_size: int = 64, query_block: int = 1, sink_blocks: int = 1, local_blocks: int = 1,
                 softmax_scale: float = 0.0, device=None):
        ext = B.load_torch()
        self.cfg = B.BlockConfig(num_q_heads=num_q_heads, num_kv_heads=num_kv_heads, head_dim_qk=head_dim_qk,
                                 head_dim_v=head_dim_v, softmax_scale=softmax_scale, block_size=block_size,
                                 query_block=query_block, max_blocks=max_blocks, sink_blocks=sink_blocks,
                                 local_blocks=local_blocks)
        B.vpp_block_attn_workspace(self.cfg, 0, 0)  # refuses a bad configuration
        dev = torch.device(device) if device is not None else torch.device("cuda")
        if dev.type != "cuda":
            raise ValueError("the plan must be on a GPU, not %s" % dev)
        self.device = dev if dev.index is not None else torch.device("cuda", torch.cuda.current_device())
        self._native = ext.Block(bytes(self.cfg), self.device.index)
        self._qb: Optional[torch.Tensor] = None
        self.tokens = self.num_query_blocks = self.workspace_bytes = self.select_bytes = 0

    # -- planning -----------------------------------------------------------
    def _not_capturing(self, what: str):
        with torch.cuda.device(self.device):
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("%s() copies from the host: call it before the capture" % what)

    def plan(self, cu_q: Sequence[int], kv_start: Sequence[int], prefix_len: Sequence[int]) -> int:
        """Cut the chunk's segments (as for ``ChunkAttention.plan``; kv_start a multiple of block_size)
        into query blocks. Returns their number. Not within a graph capture."""
        self._not_capturing("plan")
        qb = B.vpp_query_blocks(cu_q, kv_start, prefix_len, self.cfg.query_block, self.cfg.block_size)
        cu = [int(x) for x in cu_q]
        used = [s for s in range(len(kv_start)) if cu[s + 1] > cu[s]]
        self.segments = len(kv_start)
        # cache rows and positions the chunk reads, checked against the block table before every run
        self.seg_rows = max([int(kv_start[s]) + int(prefix_len[s]) + cu[s + 1] - cu[s] for s in used] or [0])
        self.max_kv_len = max([int(prefix_len[s]) + cu[s + 1] - cu[s] for s in used] or [0])
        self.tokens = cu[-1]
        self.num_query_blocks = len(qb)
        self.workspace_bytes = B.vpp_block_attn_workspace(self.cfg, len(qb), self.tokens)
        try:
            self.select_bytes = B.vpp_block_select_workspace(self.cfg, len(qb), self.max_kv_len)
        except B.VppError:  # more blocks than a selection takes: select() says so, lists of another kind run
            self.select_bytes = -1
        with torch.cuda.device(self.device):
            host = torch.empty(max(1, 8 * len(qb)), dtype=torch.int32, pin_memory=True)
            host.numpy()[:8 * len(qb)] = qb.view("<i4").reshape(-1)
            dev = torch.empty_like(host, device=self.device)
            dev.copy_(host, non_blocking=True)  # torch keeps the pinned memory until the copy is done
            self._plan_stream = torch.cuda.current_stream(self.device)
            self._copied = self._plan_stream.record_event()
        self._qb = dev
        self._native.set_plan(dev.data_ptr(), len(qb), self.tokens, self.segments, self.seg_rows, self.max_kv_len,
                              self.workspace_bytes, self.select_bytes, self._plan_stream.cuda_stream)
        return len(qb)

    def completed(self, cu_q: Sequence[int], kv_start: Sequence[int], prefix_len: Sequence[int], host_block_table,
                  page_size: int) -> torch.Tensor:
        """The blocks of the cache (int64 indices, on the GPU, copied there on the current stream) that a
        chunk completes, for ``summarize``; host_block_table is a host copy of the block table (array
        [segments, pages_per_row]). Not within a graph capture."""
        self._not_capturing("completed")
        ids = B.vpp_completed_blocks(cu_q, kv_start, prefix_len, host_block_table, page_size, self.cfg.block_size)
        return torch.from_numpy(ids).pin_memory().to(self.device, non_blocking=True)

    def new_summaries(self, num_pages: int, page_size: int) -> torch.Tensor:
        """Summaries (zeros) of a cache of num_pages pages: bf16 [num_pages, page_size / block_size, Hkv, dqk]."""
        c = self.cfg
        if page_size < c.block_size or page_size & (page_size - 1):
            raise ValueError("page_size must be a power of two of at least block_size")
        return torch.zeros(num_pages, page_size // c.block_size, c.num_kv_heads, c.head_dim_qk, dtype=torch.bfloat16,
                           device=self.device)

    # -- checks ---------------------------------------------------------------
    def _tensor(self, t: torch.Tensor, name: str, dtype, shape, contiguous: bool = False):
        if t.dtype != dtype:
            raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
        if t.device != self.device:
            raise ValueError("%s is on %s but the plan is on %s" % (name, t.device, self.device))
        if t.dim() != len(shape) or any(w is not None and h != w for h, w in zip(t.shape, shape)):
            raise ValueError("%s has shape %s, not %s" % (name, tuple(t.shape), tuple("*" if x is None else x for x in shape)))
        if contiguous and not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
        if t.shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError("%s: last dimension must be contiguous" % name)

    def _queries(self, q: torch.Tensor):
        if self._qb is None:
            raise RuntimeError("plan() must be called before select() and run_paged()")
        c = self.cfg
        self._tensor(q, "q", torch.bfloat16, (None, c.num_q_heads, c.head_dim_qk))
        if q.shape[0] < self.tokens:
            raise ValueError("q has %d rows, the plan %d" % (q.shape[0], self.tokens))

    def _table(self, block_table: torch.Tensor, page: int):
        self._tensor(block_table, "block_table", torch.int32, (None, None))
        if block_table.shape[0] < self.segments:
            raise ValueError("block_table has %d rows for %d segments" % (block_table.shape[0], self.segments))
        if self.seg_rows > block_table.shape[1] * page:
            raise ValueError("the planned chunk reads cache rows up to %d but a block-table row maps %d"
                             % (self.seg_rows, block_table.shape[1] * page))

    def _summaries(self, summaries: torch.Tensor):
        c = self.cfg
        self._tensor(summaries, "summaries", torch.bfloat16, (None, None, c.num_kv_heads, c.head_dim_qk), contiguous=True)

    def _lists(self, blocks: torch.Tensor):
        c = self.cfg
        self._tensor(blocks, "blocks", torch.int32, (self.num_query_blocks, c.num_kv_heads, c.max_blocks), contiguous=True)

    def _stream(self, stream, planned: bool = True):
        """The launch stream (default: torch's current stream), ordered behind the plan's copy. A stream
        that captures is not: the copy belongs before the capture, which torch begins with a
        synchronization."""
        s = stream if stream is not None else torch.cuda.current_stream(self.device)
        if s.device != self.device:
            raise ValueError("stream is on %s but the tensors are on %s" % (s.device, self.device))
        if planned and s != self._plan_stream:
            with torch.cuda.stream(s):
                capturing = torch.cuda.is_current_stream_capturing()
            if not capturing:
                s.wait_event(self._copied)
            self._qb.record_stream(s)
        return s

    # -- running ------------------------------------------------------------
    def summarize(self, k_pages: torch.Tensor, blocks: torch.Tensor, summaries: torch.Tensor,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Write the summaries of the listed blocks of k_pages [pages, page_size, Hkv, dqk] (bf16) into
        ``summaries`` (of ``new_summaries``); blocks: int64 indices on the GPU (``completed``), those
        outside the cache are skipped."""
        if stream is None and ChunkAttention._done(self._native.summarize(k_pages, blocks, summaries),
                                                   "vpp_block_summarize_paged"):
            return summaries
        c = self.cfg
        self._tensor(k_pages, "k_pages", torch.bfloat16, (None, None, c.num_kv_heads, c.head_dim_qk))
        self._summaries(summaries)
        if summaries.shape[0] != k_pages.shape[0] or summaries.shape[1] * c.block_size != k_pages.shape[1]:
            raise ValueError("summaries %s do not match k_pages %s" % (tuple(summaries.shape), tuple(k_pages.shape)))
        self._tensor(blocks, "blocks", torch.int64, (None,), contiguous=True)
        s = self._stream(stream, planned=False)
        with torch.cuda.device(self.device):
            B.vpp_block_summarize_paged(c, k_pages.data_ptr(), k_pages.stride(0), k_pages.stride(1), k_pages.stride(2),
                                        int(k_pages.shape[1]), int(k_pages.shape[0]), blocks.data_ptr(),
                                        int(blocks.shape[0]), summaries.data_ptr(), s.cuda_stream)
        return summaries

    def select(self, q: torch.Tensor, summaries: torch.Tensor, block_table: torch.Tensor,
               blocks: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """The lists of the planned chunk's query blocks: int32 [query blocks, Hkv, max_blocks], ascending,
        -1 in unused places (allocated when ``blocks`` is None). q [tokens, Hq, dqk] as the attention
        takes it; block_table int32 [segments, pages_per_row] on the GPU."""
        if stream is None and blocks is not None and ChunkAttention._done(
                self._native.select(q, summaries, block_table, blocks), "vpp_block_select_paged"):
            return blocks
        self._queries(q)
        self._summaries(summaries)
        c = self.cfg
        page = int(summaries.shape[1]) * c.block_size
        self._table(block_table, page)
        s = self._stream(stream)
        if blocks is None:
            blocks = new_on(s, (self.num_query_blocks, c.num_kv_heads, c.max_blocks), torch.int32)
        self._lists(blocks)
        ws = new_on(s, (self.select_bytes,), torch.uint8) if self.select_bytes > 0 else None
        with torch.cuda.device(self.device):
            B.vpp_block_select_paged(c, self._qb.data_ptr(), self.num_query_blocks, q.data_ptr(), q.stride(0), q.stride(1),
                                     self.tokens, summaries.data_ptr(), page, int(summaries.shape[0]),
                                     block_table.data_ptr(), block_table.stride(0), self.segments,
                                     int(block_table.shape[1]), self.max_kv_len, blocks.data_ptr(),
                                     ws.data_ptr() if ws is not None else 0, max(0, self.select_bytes), s.cuda_stream)
        return blocks

    def run_paged(self, q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, block_table: torch.Tensor,
                  blocks: torch.Tensor, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None):
        """Attention of the planned chunk to the listed blocks (``select``, or lists of the same form). Caches,
        block table, out and lse as for ``ChunkAttention.run_paged``. Returns (out, lse)."""
        if stream is None and out is not None and ChunkAttention._done(
                self._native.run_paged(q, k_pages, v_pages, block_table, blocks, out, lse), "vpp_block_attn_run_paged"):
            return out, lse
        self._queries(q)
        c = self.cfg
        self._tensor(k_pages, "k_pages", torch.bfloat16, (None, None, c.num_kv_heads, c.head_dim_qk))
        self._tensor(v_pages, "v_pages", torch.bfloat16, tuple(k_pages.shape[:2]) + (c.num_kv_heads, c.head_dim_v))
        page = int(k_pages.shape[1])
        self._table(block_table, page)
        self._lists(blocks)
        s = self._stream(stream)
        if out is None:
            out = new_on(s, (self.tokens, c.num_q_heads, c.head_dim_v), torch.bfloat16)
        self._tensor(out, "out", torch.bfloat16, (None, c.num_q_heads, c.head_dim_v))
        if out.shape[0] < self.tokens:
            raise ValueError("out has %d rows, the plan %d" % (out.shape[0], self.tokens))
        if lse is not None:
            self._tensor(lse, "lse", torch.float32, (c.num_q_heads, None))
            if lse.shape[1] < self.tokens:
                raise ValueError("lse has %d columns, the plan %d rows" % (lse.shape[1], self.tokens))
        ws = new_on(s, (self.workspace_bytes,), torch.uint8) if self.workspace_bytes else None
        with torch.cuda.device(self.device):
            B.vpp_block_attn_run_paged(c, self._qb.data_ptr(), self.num_query_blocks, q.data_ptr(), q.stride(0), q.stride(1),
                                       self.tokens, k_pages.data_ptr(), k_pages.stride(0), k_pages.stride(1),
                                       k_pages.stride(2), v_pages.data_ptr(), v_pages.stride(0), v_pages.stride(1),
                                       v_pages.stride(2), page, int(k_pages.shape[0]), block_table.data_ptr(),
                                       block_table.stride(0), self.segments, int(block_table.shape[1]),
                                       blocks.data_ptr(), out.data_ptr(), out.stride(0), out.stride(1),
                                       lse.data_ptr() if lse is not None else 0, lse.stride(0) if lse is not None else 0,
                                       ws.data_ptr() if ws is not None else 0, self.workspace_bytes, s.cuda_stream)
        return out, lse
