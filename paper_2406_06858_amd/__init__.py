"""MI355X-native fused tensor-parallel GEMMs (GEMM-ReduceScatter, AllGather-GEMM).

The compute path is two C-ABI libraries built from `csrc/`: `binding` marshals arguments to the fused
GEMMs', `ffn`, `norm` and `loss` to the one with the gated feed-forward and 4-bit operators, the
root-mean-square norm and the cross entropy.  Importing the package does not load them; the first call does, and raises if the
library has not been built.
"""
__all__ = ["binding", "ffn", "inputs", "loss", "norm"]
