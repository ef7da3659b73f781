"""B200-native half-precision GEMM (C = A * B^T, fp16 in, fp32 accumulate, fp16 out).

``paper_2512_02551_b200.hgemm`` is the thin ctypes binding of the C-ABI library built
from ``csrc/``; ``paper_2512_02551_b200.inputs`` draws the seeded synthetic workloads.  ``fp8`` binds the 8-bit products with
block scales (dense and over experts) and their quantiser, ``fp4`` the 4-bit ones, ``routing`` the routing of tokens to experts,
``few_tokens`` the layer of experts of a decoding step; ``run_experts`` puts them together in a layer of experts.
"""
__all__ = ["hgemm", "inputs", "build", "fp8", "fp4", "few_tokens", "routing"]
