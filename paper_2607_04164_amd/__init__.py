"""MI355X-native grouped ("full-brownout") MoE layer forward.

The work runs in ``libbrownout_moe.so`` (HIP kernels for gfx950) behind the C
ABI in ``include/brownout_moe.h``; this package holds its build step, a thin
ctypes binding and the seeded workload generator used by tests and benchmarks.
"""
from .binding import (BMOE_BF16, BMOE_F32, W4, BmoeError, Desc, LayerForward, ResidualBlock, combine, dispatch,
                      ffn, ffn_down, ffn_gate_up, load_library, make_desc, new_dispatch_workspace, post_norm,
                      pre_norm, route, validate, validate_map, w4_ffn, w4_gate_up, w4_matmul, w4_quantize,
                      workspace_bytes)

__all__ = ["BMOE_BF16", "BMOE_F32", "BmoeError", "Desc", "LayerForward", "ResidualBlock", "W4", "combine", "dispatch",
           "ffn", "ffn_down", "ffn_gate_up", "load_library", "make_desc", "new_dispatch_workspace", "post_norm",
           "pre_norm", "route", "validate", "validate_map", "w4_ffn", "w4_gate_up", "w4_matmul", "w4_quantize",
           "workspace_bytes"]
