"""libmsda: multi-scale deformable attention (MSDA) forward and backward for AMD MI355X (gfx950),
and the operators around it in a transformer layer: layer norm, rotary positions and dense attention; at inference in
8 bits root-mean-square norm, products of 8-bit integers, and a paged cache with the attention that reads it.

The compute path is the C-ABI library ``libmsda.so`` (hand-written HIP kernels); the Python
module :mod:`paper_2505_14022_amd.msda` is a thin ctypes binding over it. Importing this
package loads nothing; the library is loaded on first use and a missing library is an error.
"""

__all__ = ["msda", "workloads"]
