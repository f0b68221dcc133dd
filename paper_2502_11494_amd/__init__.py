"""DART token reduction (arXiv 2502.11494, Section 3.3) for MI355X: hand-written
HIP kernels behind the C ABI of include/dart.h, with a ctypes binding."""
from .binding import (DART_BF16, DART_ERR_ALIGN, DART_ERR_BUDGET, DART_ERR_DEVICE,  # noqa: F401
                      DART_ERR_DTYPE, DART_ERR_HIP, DART_ERR_NULL, DART_ERR_SHAPE,
                      DART_ERR_STATIC_LIMIT,
                      DART_ERR_WORKSPACE, DART_F32, DART_OK, DART_PIVOT_MAX_L1,
                      DART_PIVOT_GIVEN, DART_PIVOT_MIN_L1, DART_PIVOT_RANDOM, DART_SCORE_MAX, DART_SCORE_MIN,
                      DART_SCORE_PER_PIVOT, DartCache, DartDesc, DartError, DartEviction, DartRotation, DartRowTensor,
                      alloc_attend_4bit_workspace, alloc_attend_weights_workspace, alloc_attend_workspace,
                      alloc_evict_workspace, alloc_pool_4bit, alloc_workspace, dart_append_4bit, dart_attend,
                      dart_attend_4bit, dart_attend_4bit_workspace_bytes, dart_attend_weights,
                      dart_attend_weights_workspace_bytes, dart_evict, dart_evict_most, dart_evict_workspace_bytes,
                      dart_read_4bit, make_cache_4bit, make_eviction, dart_attend_workspace_bytes,
                      dart_compact_sequences,
                      dart_device_status, dart_duplication_scores, dart_gather_compact,
                      dart_device_status_static, dart_probe_mfma_dot32, dart_reduce,
                      dart_reduce_profiled, dart_reduce_static, dart_reduce_with_norms,
                      dart_norm_rotate, dart_norm_rotate_append, dart_score_tile_shape,
                      dart_score_tile_shape_first_read,
                      dart_select_pivots,
                      dart_static_scratch_bytes, dart_topk_keep,
                      dart_workspace_bytes, make_cache, make_desc, make_rotation, score_tolerance, strerror)
