"""MI355X-native speculative decoding rounds for patch-autoregressive time-series transformers.

The product is the C-ABI library `libtsd.so` (declared in include/tsd.h, implemented as HIP
kernels for gfx950).  This package is its thin Python binding: argument marshalling only.
"""
from .binding import (  # noqa: F401
    TSD_BF16, TSD_DRAFT, TSD_F32, TSD_FLAG_NAIVE_VERIFY, TSD_FLAG_NO_COMPACT, TSD_FLAG_NO_GRAPH, TSD_FLAG_NO_SKINNY, TSD_FLAG_NO_TEMPERING,
    TSD_FLAG_SAMPLE_PROPOSALS, TSD_FLAG_SCRAMBLE_PAGES, TSD_FLAG_THRESHOLD_RULE, TSD_FLAG_BATCH_SYNC, TSD_FLAG_NO_PINNED_COUNTS, TSD_FLAG_NO_FUSED_DRAFT, TSD_FLAG_FUSED_DRAFT, TSD_FLAG_NO_WIDE_GEMM, TSD_FLAG_ROPE_INTERLEAVED, TSD_TARGET, TsdConfig, TsdError,
    TsdModelCfg, TsdStats, Session, accept_commit_static, bench_copy, bench_gemm, bench_mfma, lib, keep_path_static, library_path, make_config, paged_attn_static,
    rope_append_static, rope_frequencies, session_for, token_logprobs_static, tree_attn_static, verify_tokens_static, verify_tree_static, window_attn_static,
)
from . import law  # noqa: F401,E402
