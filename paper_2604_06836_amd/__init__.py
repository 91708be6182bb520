"""MI355X-native quantized Adam step of STQuant: thin Python binding over the C-ABI library.

Every step of the path runs in the HIP kernels of libstq.so; this package only marshals
arguments.  PyTorch is used by callers for device memory and streams.
"""
from .binding import (  # noqa: F401
    STQ_FLAG_STATS, STQ_FLAG_STATS_GRAD, STQ_DECIDE_R_ALG1, STQ_DECIDE_NO_DUAL, STQ_DECIDE_NO_TEMPORAL, STQ_DECIDE_NO_SPATIAL,
    STQ_F32, STQ_BF16, STQ_Q8, STQ_MAX_INNER,
    StqError, Context, Engine, Bits, HParams, LayerStats, DecideState, Matrix, Grad,
    make_matrix, make_grads, rms_norm_grad_bytes, matmul_grad_weight_bytes, cross_entropy_bytes, cross_entropy_grad_bytes,
    load_library, library_path, state_bytes, table, decide, decide_due, strerror,
)

__all__ = ["STQ_FLAG_STATS", "STQ_FLAG_STATS_GRAD", "STQ_DECIDE_R_ALG1", "STQ_DECIDE_NO_DUAL", "STQ_DECIDE_NO_TEMPORAL",
           "STQ_DECIDE_NO_SPATIAL", "decide_due", "StqError", "Context", "Engine", "Bits", "HParams", "LayerStats",
           "DecideState", "STQ_F32", "STQ_BF16", "STQ_Q8", "STQ_MAX_INNER", "Matrix", "make_matrix",
           "rms_norm_grad_bytes", "matmul_grad_weight_bytes", "cross_entropy_bytes", "cross_entropy_grad_bytes", "Grad", "make_grads",
           "load_library", "library_path", "state_bytes", "table", "decide", "strerror"]
