"""MI355X (gfx950) low-bit substitute layers of SubSpec (Sec. 4.1), the draft pass around them
(queries, keys and values from the fused projection, tree attention over a 16-bit or a 4-bit
cache, the draft-tree expansion of Sec. 4.2) and the verification of the drafted tree.

The compute path is the native library ``libsubspec.so`` (hand-written HIP,
C ABI in ``include/subspec.h``); this package only marshals arguments to it.
Importing works without a GPU; calling a device entry point needs the library
built for gfx950 and fails loudly when it is missing.
"""
from ._binding import (  # noqa: F401
    SUBSPEC_PATH_AUTO,
    SUBSPEC_PATH_GEMV,
    SUBSPEC_PATH_MFMA,
    SUBSPEC_PATH_MFMA16,
    SUBSPEC_PATH_MFMA32,
    SubspecError,
    library_path,
    load_library,
    subspec_last_error,
    subspec_qdequant,
    subspec_qlinear,
    subspec_qlinear_path,
    subspec_qlinear_noalloc,
    SUBSPEC_NOALLOC_SCRATCH_BYTES,
    subspec_qlinear_plan,
    subspec_kv4_append,
    subspec_kv4_bytes,
    subspec_kv4_read,
    subspec_qkv_rope,
    subspec_qpack,
    subspec_qpack_bytes,
    subspec_qpack_host,
    subspec_quantize,
    subspec_quantize_hqq,
    subspec_reserve,
    subspec_workspace_info,
    subspec_stack_forward,
    subspec_stack_capture,
    subspec_graph_launch,
    subspec_graph_destroy,
    subspec_tree_expand,
    Prefetcher,
    subspec_tree_attention,
    subspec_tree_attention_plan,
    subspec_tree_attention_kv4,
    subspec_tree_attention_kv4_plan,
    subspec_tree_attention_kv4_workspace_bytes,
    subspec_tree_attention_workspace_bytes,
    subspec_tree_plan,
    subspec_tree_verify,
    subspec_tree_verify_workspace_bytes,
    subspec_tree_workspace_bytes,
)
