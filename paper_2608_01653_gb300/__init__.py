"""GB300-native Hadamard-domain INT8 convolution (HaTQ's DH/WH operator).

The compute path is libhatq.so (CUDA for sm_103a, C ABI in include/hatq.h);
`hatq` is its thin ctypes binding, `chain` sequences prepared layers by a
static DH/WH profile mask, `experts` runs a feed-forward block of experts
over the token operators and `attention` an attention layer over the 4-bit
weights and the 4-bit cache.
"""
from . import build, hatq  # noqa: F401

__all__ = ["build", "hatq", "chain", "experts", "attention"]
