"""TicTac scheduling math on MI355X: recv-dependency bitsets, TIC/TAC transfer
priorities and batched makespan / scheduling-efficiency evaluation.

Sub-modules
-----------
workloads : seeded synthetic DAG and timing-sample generators (no scheduling
            arithmetic; shared by the tests of the oracle and of the GPU
            path).
binding   : ctypes binding of the C-ABI library (``libtictac.so``) built from
            ``csrc/``; everything per timing sample runs in the HIP kernels, and
            so do the dependency sets of large graphs (those of small ones
            are formed by the library's host code).
layers    : operators of a worker's layers (8-bit rows, layer norm, products
            with 8-bit weights, forward and backward) from the same library:
            the ops between the transfers.
measured  : a stack of such layers run on the GPU, its ops timed and its
            transfers ordered (``python -m paper_1803_03288_amd.measured``).
build     : compiles ``csrc/`` for gfx950 with hipcc.

Nothing is imported eagerly so that the generator module can be used on a
machine without the compiled library.
"""

__all__ = ["workloads", "binding", "layers", "measured", "build"]
