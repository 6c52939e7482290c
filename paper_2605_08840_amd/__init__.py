"""ReST-KV eviction hot path for AMD MI355X: Python binding of librestkv.so."""
from .binding import (  # noqa: F401
    LIB_PATH, RESTKV_BF16, RESTKV_F32, RESTKV_Q4, RESTKV_GROUP_MAX, RESTKV_IND_ATTENTION, RESTKV_IND_VALUE_NORM,
    RESTKV_POOL_MAX, RESTKV_TEMPORAL_INV_EMA, RESTKV_TEMPORAL_MEAN, CacheLayers, CachePages, LayerBuffers, RestkvBeams, RestkvCache, RestkvError, RestkvParams, alloc_layer_buffers,
    alloc_attend_beams_workspace, alloc_attend_workspace, alloc_beam_workspace, alloc_cache_pages, alloc_workspace, evict_layer, lib, make_beams, make_cache, make_params, restkv_append,
    restkv_attend, restkv_attend_beams, restkv_attend_beams_workspace_bytes, restkv_attend_workspace_bytes, restkv_beam_reorder,
    restkv_beam_select, restkv_beam_workspace_bytes, restkv_compact, restkv_fetch, restkv_prepare_wo, restkv_score, restkv_score_from_attention,
    restkv_score_smooth, restkv_select, restkv_select_b, restkv_select_static, restkv_select_static_capacity, restkv_smooth, restkv_smooth_b, restkv_debug_beams_list, restkv_debug_force_fp32, restkv_debug_force_shared, restkv_debug_fp32_plan, restkv_debug_score_plan,
    restkv_stream_reference, restkv_timing_enable, restkv_timing_read, restkv_version, restkv_workspace_bytes, strerror,
)
