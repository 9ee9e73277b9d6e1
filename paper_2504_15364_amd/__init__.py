"""MI355X-native KeyDiff block-prefill hot path (hand-written HIP for gfx950).

The product is ``libkeydiff.so`` (C ABI in ``include/keydiff.h``); this package
is the thin ctypes binding over it.  There is no CPU fallback: importing
``binding`` without the built library raises.
"""
from .binding import (  # noqa: F401
    ANCHOR_MEAN_KEY,
    ANCHOR_MEAN_UNIT_KEY,
    KERNEL_NAMES,
    LAYOUT_FILL,
    LAYOUT_ORDERED,
    LEFT_OUT_POSITION,
    LEFT_OUT_ROW,
    KeyDiffCache,
    KeyDiffConfig,
    KeyDiffError,
    branch_append,
    branch_attention,
    branch_chunk_attention,
    branch_chunk_workspace_bytes,
    branch_evict,
    branch_evict_workspace_bytes,
    branch_weights,
    branch_weights_workspace_bytes,
    branch_workspace_bytes,
    load_library,
    norm_rope,
    prefill_block_layers,
)
