"""MI355X linear attention (kernel a + b*x): thin Python binding over libla.so.

Every step of the computation runs in the HIP library; this package only
marshals arguments.  PyTorch is used for device memory and streams.
"""
from .binding import (EXPORTS, LA_BF16, LA_F32, LA_MAX_TRACE, LaError, la_backward,
                      la_debug_override, la_forward_static, LA_STATIC_SCRATCH_BYTES,
                      la_decode_state_bytes, la_decode_step, la_decode_prefill, la_backward_ab, la_forward_qknorm, la_backward_qknorm,
                      la_forward_qknorm_save, la_backward_qknorm_saved,
                      la_backward_saved, la_backward_traced, la_forward, la_forward_save,
                      la_forward_traced, la_saved_state_bytes, la_status_string, la_trace,
                      la_version, la_workspace_bytes, library_path, load_library)
from .binding import (LA_E4M3, LA_GATE_SIGMOID, LA_GATE_VALUE, LA_GROUP, LA_I8, la_pack_rows, la_pack_tensors, la_recurrence_backward,
                      la_recurrence_forward, la_recurrence_step, la_recurrence_workspace_bytes, la_rmsnorm_backward,
                      la_rmsnorm_forward, la_rmsnorm_workspace_bytes, la_unpack_rows)
from .binding import (LA_ACT_NONE, LA_ACT_SILU, LA_STEP_SOFTPLUS, LA_STEP_VALUE, la_conv_backward, la_conv_forward, la_conv_step,
                      la_conv_workspace_bytes, la_selective_backward, la_selective_forward, la_selective_saved_bytes,
                      la_selective_step, la_selective_workspace_bytes)

from .autograd import (LinearAttentionFunction, causal_conv, gated_recurrence, linear_attention, pack_rows, rms_norm,
                       rms_norm_quantised, selective_scan, unpack_rows)

__all__ = ["LinearAttentionFunction", "linear_attention", "LA_F32", "LA_BF16", "LA_MAX_TRACE", "EXPORTS", "LaError", "la_forward", "la_backward",
           "la_forward_traced", "la_backward_traced", "la_forward_save", "la_backward_saved",
           "la_saved_state_bytes", "la_trace", "la_debug_override", "la_decode_state_bytes", "la_decode_step", "la_decode_prefill", "la_backward_ab", "la_forward_qknorm", "la_backward_qknorm", "la_forward_qknorm_save", "la_backward_qknorm_saved", "la_forward_static", "LA_STATIC_SCRATCH_BYTES", "la_workspace_bytes",
           "la_status_string", "la_version", "library_path", "load_library",
           "gated_recurrence", "rms_norm", "rms_norm_quantised", "pack_rows", "unpack_rows", "LA_E4M3", "LA_I8",
           "LA_GROUP", "LA_GATE_VALUE", "LA_GATE_SIGMOID", "la_recurrence_workspace_bytes", "la_recurrence_forward",
           "la_recurrence_backward", "la_recurrence_step", "la_pack_rows", "la_pack_tensors", "la_unpack_rows",
           "la_rmsnorm_workspace_bytes", "la_rmsnorm_forward", "la_rmsnorm_backward",
           "causal_conv", "selective_scan", "LA_ACT_NONE", "LA_ACT_SILU", "LA_STEP_VALUE", "LA_STEP_SOFTPLUS",
           "la_conv_workspace_bytes", "la_conv_forward", "la_conv_backward", "la_conv_step", "la_selective_workspace_bytes",
           "la_selective_saved_bytes", "la_selective_forward", "la_selective_backward", "la_selective_step"]
