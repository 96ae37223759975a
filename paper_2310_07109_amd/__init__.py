"""SparseCoder hot path on MI355X: sliding-window + global sparse attention fused
with learned token pruning (arXiv 2310.07109), as hand-written gfx950 kernels
behind a C ABI (``include/sc.h`` and, for the operators of the encoder block beside
the attention, ``include/sc_block.h`` and ``include/sc_layer.h``; ``libsc.so``).

This package is the thin Python binding: it marshals torch device tensors to
the C entry points of the same names.  torch only allocates device memory and
provides the stream; every step of the path runs in the library's kernels.
There is no fallback: without the built library every call raises.
"""
from ._binding import (SC_BF16, SC_F32, SC_SCORE_FROM_BAND_PROBS, SC_SCORE_FROM_PARTIALS, Desc, ScError,  # noqa
                       lib_path, load, sc_band_probs_size, sc_encoder_attn_stack,
                       sc_encoder_attn_stack_workspace_size, sc_encoder_stack, sc_encoder_stack_workspace_size,
                       sc_ltp_prune_compact, sc_ltp_prune_compact_workspace_size, sc_ltp_score,
                       sc_ltp_score_workspace_size, sc_ltp_soft_backward,
                       sc_ltp_soft_backward_workspace_size, sc_ltp_soft_mask, sc_profile_window_kernel, sc_profile_window_kernel_read,
                       sc_score_partials_size, sc_status_str, sc_topk_prune_compact, sc_window_attention,
                       sc_window_attention_noalloc, sc_window_attention_workspace_size, SC_NOALLOC_SCRATCH_BYTES,
                       SC_ENOSCRATCH, SC_VALID_LEN, SC_VALID_POS_RANGE, SC_VALID_POS_ORDER,
                       SC_VALID_POS_UNUSED_FIRST, debug_lib_path, load_debug, sc_validate_desc, SC_ACT_GELU, SC_ACT_NONE, SC_GATE_CHANNEL, SC_GATE_NONE,
                       SC_GATE_SEQUENCE, SC_GATE_TOKEN, SC_I8, SC_NORM_LAYER, SC_NORM_RMS, SC_ACT_SILU, SC_ROTARY_BANDS,
                       SC_ROTARY_BASE, SC_ROTARY_HALF, SC_ROTARY_INTERLEAVED, SC_ROTARY_LINEAR, SC_ROTARY_PLAIN)
from ._block import (LayerI8, LinearDesc, NormDesc, sc_block_norm, sc_block_norm_backward,  # noqa
                     sc_block_norm_backward_workspace_size, sc_encoder_stack_i8,
                     sc_encoder_stack_i8_workspace_size, sc_i8_pitch, sc_linear_i8, sc_linear_i8_workspace_size,
                     sc_quantize_rows_i8, sc_quantize_weight_i8)
from ._layer import (DropoutDesc, FfnDesc, RotaryDesc, sc_dropout, sc_gated_ffn, sc_gated_ffn_backward,  # noqa
                     sc_gated_ffn_backward_workspace_size, sc_gated_ffn_saved_size, sc_gated_ffn_workspace_size,
                     sc_rotary, sc_rotary_backward, sc_rotary_backward_workspace_size, sc_rotary_frequencies)

__all__ = [
    "SC_BF16", "SC_F32", "SC_SCORE_FROM_PARTIALS", "SC_SCORE_FROM_BAND_PROBS", "Desc", "ScError", "load",
    "lib_path", "sc_status_str", "sc_score_partials_size", "sc_band_probs_size",
    "sc_window_attention_workspace_size", "sc_window_attention", "sc_ltp_score_workspace_size", "sc_ltp_score",
    "sc_ltp_prune_compact_workspace_size", "sc_ltp_prune_compact", "sc_topk_prune_compact",
    "sc_ltp_soft_mask", "sc_ltp_soft_backward_workspace_size", "sc_ltp_soft_backward",
    "sc_encoder_attn_stack_workspace_size", "sc_encoder_attn_stack", "sc_encoder_stack_workspace_size",
    "sc_encoder_stack", "sc_profile_window_kernel", "sc_profile_window_kernel_read",
    "sc_window_attention_noalloc", "SC_NOALLOC_SCRATCH_BYTES", "SC_ENOSCRATCH", "SC_VALID_LEN",
    "SC_VALID_POS_RANGE", "SC_VALID_POS_ORDER", "SC_VALID_POS_UNUSED_FIRST", "debug_lib_path", "load_debug",
    "sc_validate_desc",
    "SC_I8", "SC_ACT_NONE", "SC_ACT_GELU", "SC_NORM_LAYER", "SC_NORM_RMS", "SC_GATE_NONE", "SC_GATE_CHANNEL",
    "SC_GATE_SEQUENCE", "SC_GATE_TOKEN", "LinearDesc", "NormDesc", "sc_i8_pitch", "sc_quantize_rows_i8",
    "sc_quantize_weight_i8", "sc_linear_i8", "sc_linear_i8_workspace_size", "sc_block_norm",
    "sc_block_norm_backward", "sc_block_norm_backward_workspace_size", "LayerI8", "sc_encoder_stack_i8",
    "sc_encoder_stack_i8_workspace_size",
    "SC_ACT_SILU", "SC_ROTARY_HALF", "SC_ROTARY_INTERLEAVED", "SC_ROTARY_PLAIN", "SC_ROTARY_LINEAR", "SC_ROTARY_BASE",
    "SC_ROTARY_BANDS", "RotaryDesc", "FfnDesc", "DropoutDesc", "sc_rotary_frequencies", "sc_rotary",
    "sc_rotary_backward", "sc_rotary_backward_workspace_size", "sc_gated_ffn", "sc_gated_ffn_workspace_size",
    "sc_gated_ffn_saved_size", "sc_gated_ffn_backward", "sc_gated_ffn_backward_workspace_size", "sc_dropout",
]
