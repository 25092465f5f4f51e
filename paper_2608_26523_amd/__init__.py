"""Chunked-prefill causal attention for AMD MI355X (gfx950).

The hot path of VPP (virtual pipeline parallelism for chunked prefill): a chunk
of C query tokens at prefix offset p attends causally to the p cached prefix
tokens plus itself. Beside it, what a layer does to the same rows and cache: rotary
positions, alone and on the way into a paged cache, and attention to selected
blocks of the cache. The arithmetic runs in hand-written HIP kernels behind the C
ABI of include/; this package holds the ctypes binding, thin torch wrappers
(device memory and streams only) and the workload registry.
"""
from . import binding  # noqa: F401
from . import workloads  # noqa: F401

__all__ = ["binding", "workloads", "ChunkAttention", "Rotary", "BlockSparseAttention"]


def __getattr__(name):
    if name == "ChunkAttention":
        from .attention import ChunkAttention
        return ChunkAttention
    if name == "Rotary":
        from .rotary import Rotary
        return Rotary
    if name == "BlockSparseAttention":
        from .sparse import BlockSparseAttention
        return BlockSparseAttention
    raise AttributeError(name)
