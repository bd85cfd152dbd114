"""B200-native TOVA decode step: bounded multi-state attention with eviction.

The product is the CUDA library behind include/tova.h; this package holds its
sources (csrc/), the in-tree build, a ctypes binding with the same names, and
the seeded synthetic workloads.
"""
from .binding import (TOVA_DTYPE_BF16, TOVA_DTYPE_FP32, TOVA_FORMAT_E4M3, TOVA_FORMAT_INT8, TOVA_FORMAT_PLAIN,
                      TOVA_POLICY_H2O_HEAD, TOVA_POLICY_H2O_LAYER, TOVA_POLICY_TOVA, TOVA_POLICY_TOVA_HEAD,
                      TOVA_POLICY_WINDOW, TOVA_POS_AUTO, TOVA_ROPE_BANDS, TOVA_ROPE_HALF, TOVA_ROPE_INTERLEAVED,
                      TOVA_ROPE_LINEAR, TOVA_ROPE_NTK, TOVA_ROPE_PLAIN, TOVA_ROPE_YARN, TovaCache, TovaError, TovaRope,
                      lib, strerror, to_device, tova_cache_bytes, tova_config, tova_decode_step_static,
                      tova_logprobs_config, tova_packed_attention, tova_packed_config, tova_packed_workspace_bytes,
                      tova_paged_attention, tova_paged_config, tova_paged_workspace_bytes, tova_paged_write, tova_quant_config,
                      tova_quant_read, tova_quant_write, tova_rope_config, tova_token_logprobs, tova_tree_attention,
                      tova_tree_config, tova_tree_workspace_bytes, tova_verify_config, tova_verify_draft)

__all__ = ["TOVA_DTYPE_BF16", "TOVA_DTYPE_FP32", "TOVA_FORMAT_E4M3", "TOVA_FORMAT_INT8", "TOVA_FORMAT_PLAIN",
           "TOVA_POLICY_H2O_HEAD", "TOVA_POLICY_H2O_LAYER", "TOVA_POLICY_TOVA", "TOVA_POLICY_TOVA_HEAD",
           "TOVA_POLICY_WINDOW", "TOVA_POS_AUTO", "TOVA_ROPE_BANDS", "TOVA_ROPE_HALF", "TOVA_ROPE_INTERLEAVED",
           "TOVA_ROPE_LINEAR", "TOVA_ROPE_NTK", "TOVA_ROPE_PLAIN", "TOVA_ROPE_YARN", "TovaCache", "TovaError", "TovaRope",
           "lib", "strerror", "to_device", "tova_cache_bytes", "tova_config", "tova_decode_step_static",
           "tova_logprobs_config", "tova_packed_attention", "tova_packed_config", "tova_packed_workspace_bytes",
           "tova_paged_attention", "tova_paged_config", "tova_paged_workspace_bytes", "tova_paged_write",
           "tova_quant_config", "tova_quant_read", "tova_quant_write", "tova_rope_config", "tova_token_logprobs", "tova_tree_attention",
           "tova_tree_config", "tova_tree_workspace_bytes", "tova_verify_config", "tova_verify_draft"]
