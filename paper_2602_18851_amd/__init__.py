"""MI355X-native per-head spectral norms of attention interaction matrices
(implicit power iteration, implicit GQA) and the per-layer FP8 E4M3 scale
of arXiv 2602.18851, behind a C ABI (include/spectral.h)."""

from .spectral import (  # noqa: F401
    EXPORTED,
    AutoAlpha,
    LIB_PATH,
    SN_BF16,
    SN_E4M3,
    SN_E5M2,
    SN_F32,
    SN_FLAG_GRAM,
    SN_FLAG_LAYER,
    SN_FLAG_VALU_K_SWEEP,
    SN_I8,
    Spectral,
    SpectralError,
    load_library,
    sn_attend,
    sn_cache,
    sn_heads,
    sn_matmul,
    sn_matmul_int8,
    sn_params,
    sn_rotary,
    sn_shape,
    spectral_alpha_select,
    spectral_auto_alpha,
    spectral_cache_attend,
    spectral_cache_attend_workspace_bytes,
    spectral_cache_read,
    spectral_cache_write,
    spectral_destroy,
    spectral_overflow_terms,
    spectral_slack_ratio,
    spectral_init,
    spectral_last_error,
    spectral_logits_fp8,
    spectral_logits_fp8_rotary,
    spectral_logits_workspace_bytes,
    spectral_matmul_fp8,
    spectral_matmul_fp8_kernel,
    spectral_matmul_fp8_workspace_bytes,
    spectral_matmul_int8,
    spectral_matmul_int8_kernel,
    spectral_matmul_int8_workspace_bytes,
    spectral_profile,
    spectral_profile_read,
    spectral_quantize_fp8,
    spectral_quantize_int8,
    spectral_rotary,
    spectral_rotary_frequencies,
    spectral_set_stream,
    fp8_report,
    spectral_step,
    spectral_step_layer,
    spectral_step_noalloc,
    spectral_workspace_bytes,
)

# modules that need torch, loaded with the first of their names
_TORCH = {"Fp8Matrix": "fp8_blocks", "LinearFp8": "fp8_blocks", "matmul_fp8": "fp8_blocks",
          "quantize_fp8": "fp8_blocks", "Rotary": "rotary", "Int8Matrix": "int8_rows", "matmul_int8": "int8_rows",
          "quantize_int8": "int8_rows", "Fp8Cache": "fp8_cache"}


def __getattr__(name):
    if name not in _TORCH:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    from importlib import import_module

    value = globals()[name] = getattr(import_module("." + _TORCH[name], __name__), name)
    return value
