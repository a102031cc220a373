"""MI355X-native sparse MLA decode over the OmniAttn retained set.

Thin ctypes binding over libomniattn.so (hand-written gfx950 HIP kernels behind
the C ABI in include/omniattn.h).  There is no CPU fallback: without the built
library, or without a GPU, plan/decode raise.
"""
from .binding import (  # noqa: F401
    OmniAttnError,
    Plan,
    Problem,
    omniattn_plan,
    omniattn_plan_host,
    omniattn_plan_update,
    omniattn_decode,
    omniattn_decode_timed,
    omniattn_decode_static,
    omniattn_static_scratch_bytes,
    omniattn_ring_pages,
    omniattn_ring_slot,
    omniattn_ring_append,
    decode,
    omniattn_table_extend,
    omniattn_table_release,
    omniattn_gqa_append,
    omniattn_gqa_workspace_bytes,
    omniattn_gqa_decode_workspace_bytes,
    omniattn_gqa_decode,
    gqa_decode,
    omniattn_tree_masks,
    omniattn_gqa_tree,
    gqa_tree,
    omniattn_tree_verify_workspace_bytes,
    omniattn_tree_verify,
    omniattn_gqa_keep,
    omniattn_table_truncate,
    Table,
    Gqa,
    Verify,
    lib_path,
    load_library,
    BF16,
    FP8_E4M3,
    FP32,
)
