"""Exact non-causal multi-head attention (forward and backward) for MI355X, and
the operators of a block around it: layer norm, rms norm with the residual's
addition (also to 8 bits), dropout from a counter, rotary positions with several
axes, differential attention, and attention over key blocks that a cheap score
chooses.

A thin ctypes binding over the C ABI in include/vitattn.h; it only marshals
arguments. Every step of the computation runs in the library's HIP kernels.
PyTorch is used for device memory and the current stream only. If the built
library is missing the import of a binding function raises: there is no
fallback path.
"""
from .binding import (  # noqa: F401
    LIB_PATH,
    VITATTN_BWD_ACCUMULATE_DQ,
    VITATTN_BWD_STORE_DS,
    VITATTN_NOALLOC_MAX_ROWS,
    Strides,
    VitattnError,
    agg_bwd,
    agg_fwd,
    block_bwd,
    block_fwd,
    block_means,
    block_select,
    bwd,
    bwd_dkdv,
    bwd_dkdv_ds,
    bwd_dq,
    bwd_dq_from_ds,
    bwd_noalloc,
    bwd_rowdot,
    diff_bwd,
    diff_fwd,
    dropout_fwd,
    fwd,
    layer_norm_bwd,
    layer_norm_fwd,
    library,
    merge,
    rms_norm_bwd,
    rms_norm_fp8,
    rms_norm_fwd,
    rotary_fwd,
    status_str,
    strides_of,
    ulysses_pack,
    ulysses_pack_out,
    ulysses_unpack,
    ulysses_unpack_out,
    version,
    workspace_bytes,
    workspace_bytes_kv,
)
from .autograd import attention, block_attention, diff_attention, dropout, layer_norm, rms_norm, rotary  # noqa: F401,E402
