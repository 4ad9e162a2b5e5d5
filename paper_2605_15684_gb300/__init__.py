"""GB300-native Shift Sparse Block Attention (SSBA) forward.

The compute path is the CUDA library ``libssba.so`` (hand-written sm_103a kernels
behind the C-ABI declared in ``include/ssba.h``); this package is a thin ctypes
binding over it. There is no CPU fallback: if the library is missing the calls
raise.
"""
from .api import (  # noqa: F401
    SsbaDesc, SsbaError, BoundLayer, BoundSelectLayer, backward, backward_workspace_bytes, build_mask,
    build_mask_noalloc, default_forward_workspace, forward, forward_dense, forward_fused, forward_joint,
    forward_select, forward_workspace_bytes, get_status, haar_dwt, haar_dwt_pyramid, haar_iwt, haar_iwt_pyramid,
    keep_count, library_path, load_library, mask_workspace_bytes, pool_blocks, qkv_rope_pool, realized_sparsity,
    select_mask,
)
from .cache import (  # noqa: F401
    Cache, CacheDesc, CacheStep, PagedCache, PageTable, cache_alloc, cache_append, cache_attend,
    cache_attend_workspace_bytes, cache_copy, cache_select,
)
from .layer import (  # noqa: F401
    gated_linear, gated_linear_backward, linear, linear_backward, linear_backward_workspace_bytes, rms_norm,
    rms_norm_backward, rms_norm_backward_workspace_bytes, rope_axes,
)

__all__ = [
    "SsbaDesc", "SsbaError", "BoundLayer", "BoundSelectLayer", "backward", "backward_workspace_bytes",
    "build_mask", "build_mask_noalloc", "default_forward_workspace", "forward", "forward_dense", "forward_fused",
    "forward_joint", "forward_select", "forward_workspace_bytes", "get_status", "haar_dwt", "haar_dwt_pyramid",
    "haar_iwt", "haar_iwt_pyramid", "keep_count", "library_path", "load_library", "mask_workspace_bytes",
    "pool_blocks", "qkv_rope_pool", "realized_sparsity", "select_mask",
    "Cache", "CacheDesc", "CacheStep", "PagedCache", "PageTable", "cache_alloc", "cache_append", "cache_attend", "cache_attend_workspace_bytes",
    "cache_copy", "cache_select",
    "gated_linear", "gated_linear_backward", "linear", "linear_backward", "linear_backward_workspace_bytes", "rms_norm",
    "rms_norm_backward", "rms_norm_backward_workspace_bytes", "rope_axes",
]
