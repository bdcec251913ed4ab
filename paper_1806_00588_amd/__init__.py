"""MI355X-native LSH reduced-vocabulary softmax + beam expansion (thin binding over the C ABI).

Every step of the path runs in the HIP kernels of liblshbeam.so; this package only marshals
arguments.  PyTorch is used for device memory and streams, nothing else.  There is no CPU
fallback: if the library is missing or no GPU is present the calls raise.
"""
from .binding import (CachePool, LshBeamError, PackedWeights, Tables, attention_params, attention_workspace_bytes, beam_select, build_tables,
                      cache_advance, cache_attention, cache_params, cache_workspace_bytes, cache_write, decode_step, delta_params, delta_rule,
                      delta_workspace_bytes, kernel_names, load_library, library_path, packed_gated, packed_linear, packed_params,
                      packed_quantize, packed_values, packed_workspace_bytes, select_params, select_workspace_bytes,
                      step_workspace_bytes)

__all__ = ["CachePool", "LshBeamError", "PackedWeights", "Tables", "attention_params", "attention_workspace_bytes", "beam_select",
           "build_tables", "cache_advance", "cache_attention", "cache_params", "cache_workspace_bytes", "cache_write",
           "decode_step", "delta_params", "delta_rule", "delta_workspace_bytes", "kernel_names", "load_library", "library_path",
           "packed_gated", "packed_linear", "packed_params", "packed_quantize", "packed_values", "packed_workspace_bytes",
           "select_params", "select_workspace_bytes", "step_workspace_bytes"]
