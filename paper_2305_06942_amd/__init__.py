"""Fused embedding-bag pooling + All-to-All send layout, and fused GEMV +
AllReduce, for MI355X (gfx950); the router, tokens sorted by expert, and
products with 4-bit and 8-bit weights, for layers built of experts.

Python binding of the C ABI in ``include/ebag_a2a.h`` and ``gemv_ar.h`` (argument marshalling
only: every step of the operation runs in the HIP library
``libebag_a2a.so`` built next to this file).  There is no fallback: if the
library is missing, :func:`load` raises.
"""
from .abi import (EBAG_BF16, EBAG_F16, EBAG_F32, EbagError, GemvAR, MoePerm, Plan, Q4Gemv, Q8Gemv,  # noqa: F401
                  default_opts, forward_noalloc, gemv_default_opts, last_error, load, queue_stream, queue_stream_destroy, symbols)
