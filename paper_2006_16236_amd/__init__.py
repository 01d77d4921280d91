"""MI355X-native linear attention (arXiv 2006.16236): the hand-written gfx950
kernels behind the C ABI of include/la.h, and a thin ctypes binding.

Importing this package loads libla_hip.so; there is no fallback if it is absent.
"""
from .binding import (LA_BF16, LA_F32, LA_F32_POLY2, LaError, la_causal_bwd, la_causal_bwd_bnhd, la_causal_bwd_state, la_causal_bwd_workspace,
                      la_causal_fwd, la_causal_fwd_bnhd, la_causal_fwd_noalloc, la_causal_fwd_state, la_causal_fwd_workspace, la_global_bwd, la_global_bwd_bnhd, la_global_bwd_workspace, la_global_fwd, la_global_fwd_bnhd,
                      la_global_fwd_workspace, la_kernel_name, la_profile_begin, la_profile_end,
                      la_recurrent_step, la_recurrent_steps, la_tuning_reload, la_version, status_string)

from .layer import (la_conv_bwd, la_conv_bwd_workspace, la_conv_fwd, la_conv_step, la_norm_bwd, la_norm_bwd_workspace, la_norm_fwd,
                    la_scan_bwd, la_scan_bwd_workspace, la_scan_fwd, la_scan_fwd_workspace, la_scan_step)

from .autograd import causal_conv, causal_linear_attention, layer_norm, linear_attention, selective_scan

__all__ = ["causal_conv", "causal_linear_attention", "layer_norm", "linear_attention", "selective_scan", "LA_BF16", "LA_F32", "LA_F32_POLY2", "LaError", "la_causal_bwd", "la_causal_bwd_bnhd", "la_causal_bwd_state", "la_causal_bwd_workspace",
           "la_causal_fwd", "la_causal_fwd_bnhd", "la_causal_fwd_noalloc", "la_causal_fwd_state", "la_causal_fwd_workspace", "la_global_bwd", "la_global_bwd_bnhd", "la_global_bwd_workspace", "la_global_fwd", "la_global_fwd_bnhd", "la_global_fwd_workspace",
           "la_kernel_name", "la_profile_begin", "la_profile_end", "la_recurrent_step", "la_recurrent_steps", "la_tuning_reload", "la_version",
           "status_string", "la_conv_bwd", "la_conv_bwd_workspace", "la_conv_fwd", "la_conv_step", "la_norm_bwd", "la_norm_bwd_workspace",
           "la_norm_fwd", "la_scan_bwd", "la_scan_bwd_workspace", "la_scan_fwd", "la_scan_fwd_workspace", "la_scan_step"]
