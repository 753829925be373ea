"""solfp4: NVFP4 linear layer (quantize, block-scaled GEMM, linear) for
AMD MI355X, plus its MXFP4 variant on the native scaled FP4 matrix
instructions, and the operators around it (root-mean-square and layer norm
with the residual's addition, low-rank adapters beside a linear, the backward
passes of these, rotary positions, linears of few tokens with 4-bit weights),
as a C-ABI HIP library with a thin Python binding.

The binding (and so libsolfp4.so) loads on first use of any name below and
raises ImportError if the library has not been built.
"""
_NAMES = ("EXPORTED", "LIB_PATH", "Solfp4Error", "lib", "gemm_plan", "FORMAT_NVFP4",
          "FORMAT_MXFP4", "nvfp4_gemm",
          "nvfp4_gemm_workspace_bytes", "nvfp4_linear", "nvfp4_linear_workspace_bytes",
          "nvfp4_quantize", "nvfp4_gelu_amax", "nvfp4_quantize_amax", "nvfp4_quantize_encode", "nvfp4_quantize_noalloc", "nvfp4_quantize_workspace_bytes", "mxfp4_gemm", "mxfp4_linear", "mxfp4_linear_workspace_bytes", "mxfp4_quantize",
          "add_rmsnorm", "mxfp8_add_rmsnorm", "mxfp4_add_rmsnorm", "rmsnorm_backward",
          "rmsnorm_backward_workspace_bytes", "add_layernorm", "mxfp8_add_layernorm",
          "mxfp4_add_layernorm", "layernorm_backward", "layernorm_backward_workspace_bytes", "rotary", "rotary_frequencies", "rotary_table",
          "nvfp4_weight_linear", "mxfp4_weight_linear", "mxfp8_linear",
          "AdapterPlan", "adapter_plan", "adapter_plan_bytes", "add_adapters",
          "add_adapters_workspace_bytes", "adapters_backward", "adapters_backward_workspace_bytes")
__all__ = list(_NAMES)


def __getattr__(name):
    if name in _NAMES:
        from . import _binding
        # found once: a call through the package costs no lookup here afterwards
        value = globals()[name] = getattr(_binding, name)
        return value
    raise AttributeError(name)
