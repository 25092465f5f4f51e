"""Rotary positions: the torch-facing wrapper of include/vpp_rope.h.

``Rotary`` holds how a model's heads are rotated -- which dims, in which pairs, at which
frequencies, stretched for long contexts or not -- and rotates rows (``rotate``), or a chunk's
queries and keys on the way into a paged cache (``append_paged``), which takes the place of
``kv_append_paged`` and two rotations. The arithmetic runs in the HIP library; there is no
other implementation to fall back to.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as B
from .attention import ChunkAttention


def frequencies(rotary_dim: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                original_len: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0,
                low_factor: float = 1.0, high_factor: float = 4.0):
    """(radians per position of each pair, factor on the rotated values) of a scaling:

    * ``None``: base ** (-2 i / rotary_dim);
    * ``"linear"``: those divided by factor (positions interpolated);
    * ``"ntk"``: the base raised so that the slowest pair turns factor times more slowly;
    * ``"yarn"``: pairs that turn more than beta_fast times within original_len as they are, those that
      turn less than beta_slow times divided by factor, a ramp over the pair's index between;
      rotated values times 0.1 ln(factor) + 1;
    * ``"bands"``: pairs that turn more than high_factor times within original_len as they are, those
      that turn less than low_factor times divided by factor, a ramp over the turns between.
    """
    if rotary_dim < 16 or rotary_dim % 16:
        raise ValueError("rotary_dim must be a multiple of 16, got %d" % rotary_dim)
    if not (math.isfinite(base) and base > 1 and math.isfinite(factor) and factor > 0):
        raise ValueError("base must be finite and above 1, factor finite and above 0")
    i = np.arange(rotary_dim // 2, dtype=np.float64)
    if scaling == "ntk":
        base = base * factor ** (rotary_dim / (rotary_dim - 2.0))
    f = base ** (-2.0 * i / rotary_dim)
    if scaling in (None, "ntk"):
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling not in ("yarn", "bands"):
        raise ValueError("unknown scaling %r" % (scaling,))
    if original_len < 1:
        raise ValueError("scaling %r needs original_len, the length that the model was trained on" % scaling)
    if scaling == "yarn":
        if not beta_fast > beta_slow > 0:
            raise ValueError("beta_fast must be above beta_slow, and that above 0")
        low, high = (rotary_dim * math.log(original_len / (turns * 2 * math.pi)) / (2 * math.log(base))
                     for turns in (beta_fast, beta_slow))
        low, high = max(math.floor(low), 0), min(math.ceil(high), rotary_dim - 1)
        slow = np.clip((i - low) / max(high - low, 0.001), 0.0, 1.0)
        return f / factor * slow + f * (1.0 - slow), 0.1 * math.log(factor) + 1.0
    if not high_factor > low_factor > 0:
        raise ValueError("high_factor must be above low_factor, and that above 0")
    slow = 1.0 - np.clip((original_len * f / (2 * math.pi) - low_factor) / (high_factor - low_factor), 0.0, 1.0)
    return f / factor * slow + f * (1.0 - slow), 1.0


def new_on(stream: torch.cuda.Stream, shape, dtype) -> torch.Tensor:
    """A tensor that work on ``stream`` writes first: of memory that was last used there, and kept
    for what the current stream does with it after."""
    cur = torch.cuda.current_stream(stream.device)
    if stream == cur:
        return torch.empty(shape, dtype=dtype, device=stream.device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=stream.device)
    t.record_stream(cur)
    return t


class Rotary:
    """How heads of ``head_dim`` dims are rotated.

    ``rotary_dim`` dims (default: all from ``offset`` on) are rotated, in pairs (i, i + rotary_dim / 2)
    (``layout="half"``) or (2i, 2i + 1) (``"interleaved"``); the others are copied. The angles
    per position are those of :func:`frequencies`, or ``freq`` (radians, one a pair) with
    ``scale`` on the rotated values. Positions are int64, any size: angles are exact.
    """

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, offset: int = 0, layout: str = "half",
                 base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0, original_len: int = 0,
                 freq: Optional[Sequence[float]] = None, scale: Optional[float] = None, device=None, **ramp):
        if layout not in ("half", "interleaved"):
            raise ValueError("layout must be 'half' or 'interleaved', got %r" % (layout,))
        rotary_dim = head_dim - offset if rotary_dim is None else rotary_dim
        if head_dim < 16 or head_dim % 8 or head_dim > 1024 or offset < 0 or offset % 8 or rotary_dim < 16 \
                or rotary_dim % 16 or offset + rotary_dim > head_dim:
            raise ValueError("%d dims from %d on of %d cannot be rotated: head_dim and offset are multiples of 8 "
                             "(head_dim at most 1024), rotary_dim of 16" % (rotary_dim, offset, head_dim))
        if freq is None:
            freq, s = frequencies(rotary_dim, base, scaling, factor, original_len, **ramp)
            scale = s if scale is None else scale
        elif scaling is not None or ramp:
            raise ValueError("pass freq or a scaling, not both")
        self.freq = np.ascontiguousarray(np.asarray(freq, dtype=np.float64))
        if self.freq.shape != (rotary_dim // 2,):
            raise ValueError("freq must hold %d angles, one a pair" % (rotary_dim // 2))
        self.scale = 1.0 if scale is None else float(scale)
        if not math.isfinite(self.scale):
            raise ValueError("scale must be finite")
        dev = torch.device(device) if device is not None else torch.device("cuda")
        if dev.type != "cuda":
            raise ValueError("the frequencies must be on a GPU, not %s" % dev)
        ext = B.load_torch()
        turns = B.vpp_rope_turns(self.freq)
        self.device = dev if dev.index is not None else torch.device("cuda", torch.cuda.current_device())
        self.cfg = B.RopeConfig(head_dim=head_dim, rotary_dim=rotary_dim, offset=offset,
                                interleaved=int(layout == "interleaved"), scale=self.scale)
        self._turns = torch.from_numpy(turns.view(np.int64)).to(self.device)
        self._native = ext.Rope(bytes(self.cfg), self._turns.data_ptr(), self.device.index)

    # -- checks ---------------------------------------------------------------
    def _rows(self, t: torch.Tensor, name: str, shape):
        ChunkAttention._check(t, name, torch.bfloat16, len(shape))
        if t.device != self.device:
            raise ValueError("%s is on %s but the frequencies are on %s" % (name, t.device, self.device))
        if any(want is not None and have != want for have, want in zip(t.shape, shape)):
            raise ValueError("%s has shape %s, not %s" % (name, tuple(t.shape), tuple("*" if x is None else x for x in shape)))

    def _vector(self, t: torch.Tensor, name: str, n: int):
        if t.dtype != torch.int64 or t.dim() != 1 or t.shape[0] != n or t.device != self.device \
                or (n > 1 and t.stride(0) != 1):
            raise ValueError("%s must be a contiguous int64 vector of %d on %s" % (name, n, self.device))

    def _stream(self, stream):
        """The launch stream (default: torch's current stream)."""
        s = stream if stream is not None else torch.cuda.current_stream(self.device)
        if s.device != self.device:
            raise ValueError("stream is on %s but the tensors are on %s" % (s.device, self.device))
        self._turns.record_stream(s)
        return s

    # -- calls ----------------------------------------------------------------
    def rotate(self, x: torch.Tensor, positions: torch.Tensor, out: Optional[torch.Tensor] = None,
               inverse: bool = False, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Rotate x [tokens, heads, head_dim] (bf16) of tokens at positions [tokens] (int64, on the GPU)
        into ``out`` (allocated when None; x itself rotates in place). ``inverse`` rotates back:
        the gradient of a rotation is the inverse one of the gradient (with the same scale)."""
        if stream is None:
            res = torch.empty_like(x, memory_format=torch.contiguous_format) if out is None else out
            if ChunkAttention._done(self._native.rotate(x, positions, res, bool(inverse)), "vpp_rope"):
                return res
        self._rows(x, "x", (None, None, self.cfg.head_dim))
        s = self._stream(stream)
        if out is None:
            out = new_on(s, x.shape, torch.bfloat16)
        self._rows(out, "out", tuple(x.shape))
        self._vector(positions, "positions", x.shape[0])
        if x.numel():
            with torch.cuda.device(self.device):
                B.vpp_rope(self.cfg, x.data_ptr(), x.stride(0), x.stride(1), out.data_ptr(), out.stride(0), out.stride(1),
                           x.shape[0], x.shape[1], self._turns.data_ptr(), positions.data_ptr(), int(inverse),
                           s.cuda_stream)
        return out

    def append_paged(self, q: Optional[torch.Tensor], k_new: torch.Tensor, v_new: torch.Tensor,
                     k_pages: torch.Tensor, v_pages: torch.Tensor, slot_mapping: torch.Tensor,
                     positions: torch.Tensor, q_out: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> Optional[torch.Tensor]:
        """Rotate a chunk's queries q [tokens, Hq, head_dim] into ``q_out`` (allocated when None; q itself
        rotates in place) and its keys k_new [tokens, Hkv, head_dim] by ``positions``, and write the
        rotated keys and v_new [tokens, Hkv, dv] to slot_mapping [tokens] of the paged caches (as
        ``kv_append_paged``). Without queries (q None) returns None, else the rotated ones."""
        if stream is None:
            res = torch.empty_like(q, memory_format=torch.contiguous_format) if q is not None and q_out is None else q_out
            if ChunkAttention._done(self._native.append(q, k_new, v_new, k_pages, v_pages, slot_mapping, positions, res),
                                    "vpp_rope_append_paged"):
                return res
        d = self.cfg.head_dim
        self._rows(k_new, "k_new", (None, None, d))
        T, H = k_new.shape[:2]
        self._rows(v_new, "v_new", (T, H, None))
        dv = v_new.shape[2]
        self._rows(k_pages, "k_pages", (None, None, H, d))
        self._rows(v_pages, "v_pages", tuple(k_pages.shape[:2]) + (H, dv))
        self._vector(slot_mapping, "slot_mapping", T)
        self._vector(positions, "positions", T)
        s = self._stream(stream)
        if q is not None:
            self._rows(q, "q", (T, None, d))
            if q_out is None:
                q_out = new_on(s, q.shape, torch.bfloat16)
            self._rows(q_out, "q_out", tuple(q.shape))
        elif q_out is not None:
            raise ValueError("q_out without q")
        if T == 0:
            return q_out
        io = (q.data_ptr(), q.stride(0), q.stride(1), q_out.data_ptr(), q_out.stride(0), q_out.stride(1)) \
            if q is not None and q.shape[1] else (0, 0, 0, 0, 0, 0)
        with torch.cuda.device(self.device):
            B.vpp_rope_append_paged(self.cfg, *io, k_new.data_ptr(), k_new.stride(0), k_new.stride(1),
                                    v_new.data_ptr(), v_new.stride(0), v_new.stride(1),
                                    k_pages.data_ptr(), k_pages.stride(0), k_pages.stride(1), k_pages.stride(2),
                                    v_pages.data_ptr(), v_pages.stride(0), v_pages.stride(1), v_pages.stride(2),
                                    T, q.shape[1] if q is not None else 0, H, dv, int(k_pages.shape[1]),
                                    int(k_pages.shape[0]), self._turns.data_ptr(), positions.data_ptr(),
                                    slot_mapping.data_ptr(), s.cuda_stream)
        return q_out
