"""B200-native S2D2 decode step: thin Python binding over the C ABI in
include/s2d2.h.  Importing the package does not load the CUDA library; creating
an ``Engine`` does, and fails loudly if the library is missing."""
from .binding import (  # noqa: F401
    DraftStats,
    Engine,
    PagedKV,
    Rope,
    RoutePolicy,
    Rows,
    S2D2Error,
    StepResult,
    gemm_bf16_noalloc,
    kv_append,
    library_path,
    load_library,
    mxfp4_dequantize,
    mxfp4_gemm,
    mxfp4_quantize,
    mxfp4_score,
    mxfp4_score_workspace,
    mxfp4_sizes,
    ops_status,
    paged_attention,
    paged_attention_workspace,
    qk_rope,
    rope_frequencies,
    score_logits,
)
