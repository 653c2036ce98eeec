"""MI355X-native batched paged-KV attention with per-request segment masks.

The computation lives in ``libmstar_attn.so`` (HIP kernels for gfx950 and a
host planner behind the C-ABI in ``include/mstar_attn.h`` and
``include/mstar_cache.h``); ``attn`` and ``cache`` are their Python bindings.
Build with ``python -m paper_2606_12688_amd.build``.
"""

__all__ = ["attn", "build", "cache"]
