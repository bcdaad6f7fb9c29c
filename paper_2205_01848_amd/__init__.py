"""MI355X (gfx950) MoE layer with dynamic per-expert capacities and cached
assignments: libmoe.so (HIP kernels behind a C ABI, include/moe.h) and its
thin Python binding."""
from . import binding  # noqa: F401
from .layer import (AdamW, MoELayer, QuantizedExperts, RMSNorm, VocabLoss, quantize_rows,  # noqa: F401
                    rows_alloc_for)

__all__ = ["binding", "AdamW", "MoELayer", "QuantizedExperts", "RMSNorm", "VocabLoss", "quantize_rows",
           "rows_alloc_for"]
