"""MI355X-native NVFP4 hot path: quantizer, block-scaled FP4 GEMM, KV cache (HIP, gfx950)."""
from .binding import (LORA_RANK, KV_MAX_CHUNKS, ACT_GELU_TANH, ACT_NONE, OP_GEMM, OP_GEMM_ACT_QUANT, OP_GEMM_ACT_QUANT_GEMM, OP_GEMM_LORA, OP_LORA_DOWN, OP_KV_DEQUANT, OP_KV_QUANT, OP_KV_QUANT_4OVER6, OP_KV_QUANT_K, OP_KV_DEQUANT_GATHER, OP_QUANTIZE, OP_QUANTIZE_2D, OP_QUANTIZE_A2A, OP_QUANTIZE_RHT, OP_QUANTIZE_4OVER6, OUT_BF16,
                      OUT_F32, NVFP4Error, NVFP4Tensor, bf16_from_bits, bits_from_bf16, lib,
                      nvfp4_gemm, nvfp4_gemm_act_quant, nvfp4_gemm_lora, nvfp4_gemm_plan, nvfp4_lora_down, nvfp4_kv_dequant, nvfp4_kv_quant, nvfp4_kv_quant_4over6, nvfp4_kv_quant_noalloc, NOALLOC_MAX_ELEMENTS, nvfp4_kv_quant_k, nvfp4_kv_dequant_gather,
                      nvfp4_quantize, nvfp4_quantize_2d, nvfp4_quantize_for_all_to_all, nvfp4_quantize_rht, nvfp4_quantize_4over6, nvfp4_set_timing, nvfp4_set_timing_ops, nvfp4_timing_read, nvfp4_timing_read_all, nvfp4_workspace_bytes,
                      OP_PROBE, OP_GEMM_SCALE_OUT, nvfp4_gemm_scale_out, nvfp4_probe, nvfp4_set_sync_spin_limit, nvfp4_set_one_launch, ONE_LAUNCH_AUTO, ONE_LAUNCH_ALWAYS, ONE_LAUNCH_NEVER, PROBE_READ, PROBE_WRITE, PROBE_COPY, PROBE_MFMA, PROBE_MFMA_FLOPS_PER_ITER,
                      OP_QK_NORM_ROPE, OP_QK_NORM_ROPE_BACKWARD, OP_KV_CACHE_WRITE, OP_KV_CACHE_READ, OP_KV_ATTENTION, ROPE_MAX_AXES, HEAD_DIM_MAX, NVFP4KvCache, NVFP4Rope,
                      nvfp4_qk_norm_rope, nvfp4_qk_norm_rope_backward, nvfp4_kv_cache_write, nvfp4_kv_cache_read, nvfp4_kv_attention, nvfp4_kv_attention_workspace_bytes,
                      ACT_SILU, E4M3_BLOCK, OP_E4M3_QUANTIZE, OP_E4M3_QUANTIZE_2D, OP_E4M3_GEMM, OP_E4M3_GEMM_GATED, OP_GATED_BACKWARD, OP_RMS_NORM, OP_RMS_NORM_BACKWARD,
                      E4M3Tensor, nvfp4_e4m3_quantize, nvfp4_e4m3_quantize_2d, nvfp4_e4m3_gemm, nvfp4_e4m3_gemm_gated, nvfp4_gated_backward, nvfp4_rms_norm,
                      nvfp4_rms_norm_backward)
