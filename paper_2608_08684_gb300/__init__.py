"""RippleKV serving hot path on GB300 (sm_103a).

Submodules:
  ripple  -- binding of the C-ABI library libripple.so (the product path): ctypes, and the
             extension module _binding for the calls of every layer and token
  synth   -- seeded synthetic inputs (no step of the method)
  serving -- per-layer decode loops between the caller's projections, in a CUDA graph:
             contiguous caches, paged caches
  build   -- in-tree build of libripple.so and _binding with nvcc/gcc

Nothing is imported eagerly, so that importing the package never loads CUDA.
"""
