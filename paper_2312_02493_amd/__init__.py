"""MI355X-native AR-Topk gradient compressor (one GPU, W simulated workers).

The compute lives in libartopk.so (hand-written HIP for gfx950) behind the C
ABI of include/artopk.h; this package only marshals arguments.  There is no CPU
fallback: using the library without the built extension raises.
"""

from .binding import (  # noqa: F401
    ARTOPK_OPT_GUESS_MIN_N, ARTOPK_OPT_LEADER_FIRST, ARTOPK_OPT_NONTEMPORAL, ARTOPK_OPT_STAGE_TILES,
    ARTOPK_OPT_SHORT_MAX_N, ARTOPK_OPT_UPDATE_TILES_MIN_N,
    ARTOPK_PRODUCTS_DEFAULT, ARTOPK_PRODUCTS_HALF, ARTOPK_PRODUCTS_SPLIT,
    ARTOPK_MAX_TOP, artopk_adamw_scratch_bytes, artopk_adamw_state_elems, artopk_tokens_scratch_bytes,
    artopk_matrices_info, artopk_matrices_scratch_bytes, artopk_norm_scratch_bytes, artopk_scratch_bytes, artopk_variance_static,
    ARTOPK_FIXED, ARTOPK_G_BF16, ARTOPK_G_F16, ARTOPK_G_F32, ARTOPK_STAR, ARTOPK_STAR_COUNTER, ARTOPK_VAR, ARTOPK_VAR_G, ARTOPK_VAR_TOPK, ArTopkError, Context,
    AdamWContext, MatrixContext, NormContext, TokenContext, exported_symbols, lib_path, load_library,
)
