"""MI355X (gfx950) decode-step library for ASR-KF-EGR (arXiv 2512.11221).

The HIP kernels and the C ABI live in libasrkf.so (csrc/, include/asrkf.h);
``_lib`` is the thin ctypes binding with the same function names.
"""
from ._lib import (AUTO, SR, WR, FR, NONE, BF16, F32, AsrkfError, load,  # noqa: F401
                   REL_ABS, REL_SOFTMAX, SCOPE_LAYER, SCOPE_TOKEN, CAND_OUTSIDE, CAND_INSIDE,
                   ROT_HALVES, ROT_PAIRS, SCALE_NONE, SCALE_LINEAR, SCALE_BANDS, SCALE_RAMP,
                   make_rotary, asrkf_rotary_table, asrkf_set_rotary, asrkf_rotate, asrkf_reserve_drafts,
                   asrkf_tree_masks, asrkf_attend_drafts, asrkf_verify_drafts, asrkf_accept_drafts,
                   make_config, asrkf_init, asrkf_prefill, asrkf_prefill_packed, asrkf_get_rows,
                   asrkf_decode_step,
                   asrkf_decode_step_static, asrkf_restore, asrkf_stats, asrkf_stats_reset, asrkf_set_timing, asrkf_timing_series, asrkf_reset,
                   asrkf_debug_delay_side, asrkf_get_state,
                   asrkf_get_seq, asrkf_get_residency, asrkf_schedule_table, asrkf_destroy,
                   asrkf_last_error)
