"""MI355X-native prefill-time KV-cache compression (score -> allocate -> select+gather).

The package is a thin binding over libflashcache.so (hand-written HIP for gfx950).
"""
from . import binding
from .binding import (  # noqa: F401
    FC_PATH_AUTO, FC_PATH_BASIS, FC_PATH_DENSE, FC_PATH_FFT, FC_PATH_RESAMPLE, FC_PATH_STREAM, Compressor, FcKvDesc, FcRotaryPlan, FlashCacheError, MxCache, PagedKV,
    allocate, append_paged, assign_pages, choose_pages, chosen_workspace, cutoff_r, decode_attention, decode_attention_chosen,
    decode_attention_paged, decode_attention_shared, decode_attention_static,
    decode_static_scratch_bytes, describe, lowpass_energy, mx_decode_attention, mx_load, mx_page_bytes, mx_store,
    page_bounds, prepare, realisation, resolve_path, rotary, rotary_plan, score, score_layer, select_gather,
    select_gather_mx, select_gather_paged, shared_workspace,
    total_budget,
    workspace_bytes, workspace_error,
)
