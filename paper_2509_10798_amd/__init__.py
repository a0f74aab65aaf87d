"""Judge Q KV-cache eviction hot path (arXiv 2509.10798, Section 4.3) for AMD MI355X.

The work is done by hand-written HIP kernels in ``libjq.so`` (sources under
``csrc/``, C ABI in ``include/jq.h``); this package is the thin Python binding.
"""
from .binding import (  # noqa: F401
    EXPORTS, STATIC_WS_BYTES, TRACE_KERNELS, TRACE_MARKS, JQError, Pages, Shape, alloc_attend_workspace, alloc_evict_weight_workspace, alloc_workspace, attend, attend_paged,
    attend_tree, attend_tree_paged, attend_workspace_bytes, compact, compact_inplace, copy_probe, evict, evict_inplace, evict_paged, evict_paged_inplace, evict_static, evict_stream,
    evict_weight, evict_weight_paged, evict_weight_workspace_bytes, hit_rate, lib, map_mse, map_mse_fused, pool, reload_knobs, replace_lightest, replace_lightest_paged, score, score_paged, select_topk,
    status_string, workspace_bytes,
)
