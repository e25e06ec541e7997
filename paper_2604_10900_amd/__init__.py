"""MI355X-native CASK compression event: HIP kernels behind a C ABI plus a thin binding."""
from .binding import (BF16, E4M3, F32, Batch, CaskError, Outputs, Pages, Params, Rows, attend, attend_paged, cache_read, cache_write,
                      compress, compress_static, compress_step, consolidate, group_diagnostics, load, mass_diagnostics,
                      partition, plan, prefix_evict, score, workspace_bytes)

__all__ = ["BF16", "E4M3", "F32", "Batch", "CaskError", "Outputs", "Pages", "Params", "Rows", "attend", "attend_paged",
           "cache_read", "cache_write", "compress", "compress_static", "compress_step", "consolidate", "group_diagnostics",
           "load", "mass_diagnostics", "partition", "plan", "prefix_evict", "score", "workspace_bytes"]
