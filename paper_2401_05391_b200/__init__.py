"""B200-native decode attention over a segment KV cache (beam-index selection fused).

``segkv``      ctypes binding of the C-ABI library (CUDA kernels for sm_100a)
``pages``      the same for the paged cache: requests that come and go, rows in 16 or 4 bits
``workloads``  seeded synthetic inputs of the evaluation shapes
``build``      compiles ``libsegkv.so`` in-tree with nvcc
"""
from . import workloads  # noqa: F401

__all__ = ["workloads", "segkv", "pages", "build"]
