"""GB300 (sm_103a) library for VGGT-Prime's compute-adaptive mixture-of-heads global
attention: router (§4.1), routing (§4.2), full / surrogate (§4.3) / mean heads, and the
Algorithm 1 block, and the streaming operators (rotary positions, paged K/V cache, causal
attention over it), behind the C ABI of include/vp.h.  ``binding`` is the ctypes layer."""
from . import binding
from .binding import (VPError, attn_dims, attn_workspace, dims, layer_weights, paged_kv,
                      rope_options, rope_turns, router_weights, surrogate_weights, to_device,
                      vp_attn_workspace_size, vp_bin_heads, vp_global_stack, vp_head_attention,
                      vp_layer_norm, vp_linear, vp_moh_global_attention, vp_paged_attention,
                      vp_prompt_attention, vp_read_device_error, vp_rope_append, vp_router,
                      vp_status_string, vp_workspace_size, workspace)

__all__ = ["binding", "VPError", "attn_dims", "attn_workspace", "dims", "layer_weights", "paged_kv",
           "rope_options", "rope_turns", "router_weights", "surrogate_weights", "to_device",
           "vp_attn_workspace_size", "vp_bin_heads", "vp_global_stack", "vp_head_attention",
           "vp_layer_norm", "vp_linear", "vp_moh_global_attention", "vp_paged_attention",
           "vp_prompt_attention", "vp_read_device_error", "vp_rope_append", "vp_router",
           "vp_status_string", "vp_workspace_size", "workspace"]
