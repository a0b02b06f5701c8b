"""Binding of the NVFP4 HIP library: argument marshalling only.

Function names mirror the C ABI in include/nvfp4.h.  torch supplies device
memory and the current stream; every step of the path runs in the library's
kernels.  The calls that launch work take their pointers and allocate what the
caller does not pass in native code (csrc/nvfp4_host.cpp); lib() is the C ABI
itself, through ctypes, and needs neither this torch nor this Python.  There is
no CPU fallback: if a shared library is missing, or the native code was built
with another torch, the entry points raise.
"""
import ctypes
import importlib.machinery
import importlib.util
import os
import re
import sysconfig

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libnvfp4_hip.so")
_HOST_PATH = os.path.join(_HERE, "_host" + sysconfig.get_config_var("EXT_SUFFIX"))
_lib = None
_host_module = None

OUT_F32, OUT_BF16 = 0, 1
ACT_NONE, ACT_GELU_TANH = 0, 1
OP_QUANTIZE, OP_KV_QUANT, OP_GEMM_ACT_QUANT, OP_GEMM, OP_KV_DEQUANT, OP_GEMM_ACT_QUANT_GEMM = 0, 1, 2, 3, 4, 5
OP_QUANTIZE_4OVER6, OP_KV_QUANT_4OVER6, OP_KV_QUANT_K, OP_KV_DEQUANT_GATHER = 6, 7, 8, 9
KV_MAX_CHUNKS = 64
NOALLOC_MAX_ELEMENTS = 1 << 32
OP_QUANTIZE_2D, OP_QUANTIZE_RHT, OP_QUANTIZE_A2A, OP_LORA_DOWN, OP_GEMM_LORA, OP_PROBE = 10, 11, 12, 13, 14, 15
OP_GEMM_SCALE_OUT = 16
OP_QK_NORM_ROPE, OP_QK_NORM_ROPE_BACKWARD, OP_KV_CACHE_WRITE, OP_KV_CACHE_READ, OP_KV_ATTENTION = 17, 18, 19, 20, 21
ROPE_MAX_AXES, HEAD_DIM_MAX = 4, 256
LORA_RANK = 128


class _CTensor(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("global_scale", ctypes.c_void_p), ("rows", ctypes.c_int64), ("K", ctypes.c_int64)]


class _CKvChunk(ctypes.Structure):
    _fields_ = [("q", _CTensor), ("row_mean_bf16", ctypes.c_void_p), ("T", ctypes.c_int64)]


class _CRope(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("freqs", ctypes.c_void_p), ("axes", ctypes.c_int64),
                ("axis_pairs", ctypes.c_int64 * ROPE_MAX_AXES), ("interleaved", ctypes.c_int32)]


class _CHeads(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("ld", ctypes.c_int64), ("weight", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("ld_out", ctypes.c_int64), ("H", ctypes.c_int64)]


class _CHeadsGrad(ctypes.Structure):
    _fields_ = [("dy", ctypes.c_void_p), ("ld_dy", ctypes.c_int64), ("x", ctypes.c_void_p), ("ld_x", ctypes.c_int64),
                ("weight", ctypes.c_void_p), ("dx", ctypes.c_void_p), ("ld_dx", ctypes.c_int64), ("dweight", ctypes.c_void_p), ("H", ctypes.c_int64)]


class _CKvCache(ctypes.Structure):
    _fields_ = [("k_codes", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("k_global", ctypes.c_void_p), ("k_mean", ctypes.c_void_p),
                ("v_codes", ctypes.c_void_p), ("v_scales", ctypes.c_void_p), ("v_global", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("page_tokens", ctypes.c_int64), ("H", ctypes.c_int64), ("d", ctypes.c_int64)]


class NVFP4Error(RuntimeError):
    pass


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise NVFP4Error(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2605_18739_amd.build` "
                "(there is no fallback path)")
        L = ctypes.CDLL(_LIB_PATH)
        c = ctypes
        vp, i64, sz = c.c_void_p, c.c_int64, c.c_size_t
        tp = c.POINTER(_CTensor)
        L.nvfp4_quantize.restype = c.c_int
        L.nvfp4_quantize.argtypes = [vp, i64, i64, i64, c.c_int, vp, tp, vp, sz, vp]
        L.nvfp4_gemm.restype = c.c_int
        L.nvfp4_gemm.argtypes = [tp, tp, vp, i64, c.c_int, vp]
        L.nvfp4_gemm_scale_out.restype = c.c_int
        L.nvfp4_gemm_scale_out.argtypes = [tp, tp, vp, i64, vp, vp, sz, vp]
        L.nvfp4_lora_down.restype = c.c_int
        L.nvfp4_lora_down.argtypes = [vp, i64, i64, i64, vp, vp, vp, sz, vp]
        L.nvfp4_gemm_lora.restype = c.c_int
        L.nvfp4_gemm_lora.argtypes = [tp, tp, vp, vp, c.c_float, vp, i64, c.c_int, vp]
        L.nvfp4_gemm_act_quant.restype = c.c_int
        L.nvfp4_gemm_act_quant.argtypes = [tp, tp, c.c_int, vp, tp, vp, vp, sz, vp]
        L.nvfp4_kv_quant.restype = c.c_int
        L.nvfp4_kv_quant.argtypes = [vp, i64, i64, i64, tp, vp, sz, vp]
        L.nvfp4_kv_quant_noalloc.restype = c.c_int
        L.nvfp4_kv_quant_noalloc.argtypes = [vp, i64, i64, i64, tp, vp]
        L.nvfp4_kv_dequant.restype = c.c_int
        L.nvfp4_kv_dequant.argtypes = [tp, vp, i64, i64, i64, vp]
        L.nvfp4_quantize_4over6.restype = c.c_int
        L.nvfp4_quantize_4over6.argtypes = [vp, i64, i64, i64, vp, tp, vp, sz, vp]
        L.nvfp4_kv_quant_4over6.restype = c.c_int
        L.nvfp4_kv_quant_4over6.argtypes = [vp, i64, i64, i64, tp, vp, sz, vp]
        L.nvfp4_quantize_for_all_to_all.restype = c.c_int
        L.nvfp4_quantize_for_all_to_all.argtypes = [vp, i64, i64, i64, i64, vp, tp, vp, sz, vp]
        L.nvfp4_quantize_rht.restype = c.c_int
        L.nvfp4_quantize_rht.argtypes = [vp, i64, i64, i64, c.c_uint32, vp, tp, vp, sz, vp]
        L.nvfp4_quantize_2d.restype = c.c_int
        L.nvfp4_quantize_2d.argtypes = [vp, i64, i64, i64, vp, tp, tp, vp, sz, vp]
        L.nvfp4_kv_quant_k.restype = c.c_int
        L.nvfp4_kv_quant_k.argtypes = [vp, i64, i64, i64, tp, vp, vp, sz, vp]
        L.nvfp4_kv_dequant_gather.restype = c.c_int
        L.nvfp4_kv_dequant_gather.argtypes = [c.POINTER(_CKvChunk), c.c_int, vp, i64, i64, vp]
        L.nvfp4_qk_norm_rope.restype = c.c_int
        L.nvfp4_qk_norm_rope.argtypes = [c.POINTER(_CHeads), c.POINTER(_CHeads), i64, i64, c.c_float, c.POINTER(_CRope), vp]
        L.nvfp4_qk_norm_rope_backward.restype = c.c_int
        L.nvfp4_qk_norm_rope_backward.argtypes = [c.POINTER(_CHeadsGrad), c.POINTER(_CHeadsGrad), i64, i64, c.c_float, c.POINTER(_CRope), vp, sz, vp]
        L.nvfp4_kv_cache_write.restype = c.c_int
        L.nvfp4_kv_cache_write.argtypes = [c.POINTER(_CKvCache), vp, i64, vp, i64, vp, i64, c.c_int, vp]
        L.nvfp4_kv_cache_read.restype = c.c_int
        L.nvfp4_kv_cache_read.argtypes = [c.POINTER(_CKvCache), vp, i64, vp, vp, vp]
        L.nvfp4_kv_cache_read_new.restype = c.c_int
        L.nvfp4_kv_cache_read_new.argtypes = [c.POINTER(_CKvCache), vp, i64, vp, vp, vp]
        L.nvfp4_kv_attention.restype = c.c_int
        L.nvfp4_kv_attention.argtypes = [vp, i64, i64, i64, c.POINTER(_CKvCache), vp, i64, vp, vp, i64, i64, c.c_float, c.c_int, i64, i64,
                                         vp, i64, c.c_int, vp, vp, sz, vp]
        L.nvfp4_kv_attention_workspace_bytes.restype = sz
        L.nvfp4_kv_attention_workspace_bytes.argtypes = [i64] * 9
        L.nvfp4_workspace_bytes.restype = sz
        L.nvfp4_workspace_bytes.argtypes = [c.c_int, i64, i64, i64]
        L.nvfp4_status_string.restype = c.c_char_p
        L.nvfp4_status_string.argtypes = [c.c_int]
        L.nvfp4_gemm_plan.restype = c.c_int
        L.nvfp4_gemm_plan.argtypes = [i64, i64, i64, c.c_char_p, sz]
        L.nvfp4_set_timing.restype = None
        L.nvfp4_set_timing.argtypes = [c.c_int]
        L.nvfp4_set_timing_ops.restype = None
        L.nvfp4_set_timing_ops.argtypes = [c.c_uint32]
        L.nvfp4_timing_read.restype = c.c_int
        L.nvfp4_timing_read.argtypes = [c.c_int, c.POINTER(c.c_int), c.POINTER(c.c_float)]
        L.nvfp4_timing_read_all.restype = c.c_int
        L.nvfp4_timing_read_all.argtypes = [c.c_int, c.POINTER(c.c_float), c.c_int]
        L.nvfp4_set_one_launch.restype = c.c_int
        L.nvfp4_set_one_launch.argtypes = [c.c_int]
        L.nvfp4_set_sync_spin_limit.restype = None
        L.nvfp4_set_sync_spin_limit.argtypes = [c.c_uint32]
        L.nvfp4_probe.restype = c.c_int
        L.nvfp4_probe.argtypes = [c.c_int, vp, vp, sz, c.c_int, vp]
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise NVFP4Error(f"nvfp4 status {rc}: {lib().nvfp4_status_string(rc).decode()}")


def _host():
    global _host_module
    if _host_module is None:
        lib()
        if not os.path.exists(_HOST_PATH):
            raise NVFP4Error(f"{_HOST_PATH} is missing: build it with `python -m paper_2605_18739_amd.build`")
        loader = importlib.machinery.ExtensionFileLoader("_host", _HOST_PATH)
        try:
            module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_host", loader))
            loader.exec_module(module)
        except ImportError as e:
            raise NVFP4Error(f"{_HOST_PATH} does not load with torch {torch.__version__} ({e}): build it again") from e
        # torch's C++ interface changes from release to release, and not every change shows when the symbols are bound
        if module.torch_version != re.match(r"\d+(\.\d+)*", torch.__version__).group():
            raise NVFP4Error(f"{_HOST_PATH} was built with torch {module.torch_version}, this is torch {torch.__version__}: "
                             "build it again with `python -m paper_2605_18739_amd.build`")
        _host_module = module
    return _host_module


def _stream(stream=None):
    """The hipStream_t of `stream`, or of torch's current stream on the current device."""
    if stream is not None:
        return stream.cuda_stream
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _elsewhere(stream):
    """Whether `stream` is another one than torch's current stream."""
    return stream.cuda_stream != (_stream() if torch.cuda.is_initialized() else 0)


def _on(stream, call, *args):
    """The call with `stream` as torch's current stream.  What it allocates comes from that stream's pool: a block of
    the current stream's pool may still be in use by work queued there, and a workspace would go back to that pool while
    `stream` still uses it.  New outputs are noted as used by the caller's stream too, which is where they are read."""
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream)
    here = torch.cuda.current_stream(stream.device)
    with torch.cuda.stream(stream):
        result = call(*args)
    for new in result if isinstance(result, tuple) else () if isinstance(result, NVFP4KvCache) else (result,):
        if new is not None and not any(new is a for a in args):
            for t in (new.codes, new.scales, new.global_scale) if isinstance(new, NVFP4Tensor) else (new,):
                t.record_stream(here)
    return result


class NVFP4Tensor:
    """Device NVFP4 tensor: codes [rows, K/2] u8, scales [rows, K/16] u8, global_scale [1] f32."""

    def __init__(self, rows, K, device="cuda", codes=None, scales=None, global_scale=None):
        self.rows, self.K = int(rows), int(K)
        if codes is None and scales is None and global_scale is None and isinstance(device, torch.device):
            self.codes, self.scales, self.global_scale = _host().buffers(self.rows, self.K, device)
            return
        self.codes = codes if codes is not None else torch.empty((rows, K // 2), dtype=torch.uint8, device=device)
        self.scales = scales if scales is not None else torch.empty((rows, K // 16), dtype=torch.uint8, device=device)
        self.global_scale = (global_scale if global_scale is not None
                             else torch.empty(1, dtype=torch.float32, device=device))

    def c(self):
        return _CTensor(self.codes.data_ptr(), self.scales.data_ptr(), self.global_scale.data_ptr(),
                        self.rows, self.K)

    @staticmethod
    def from_host(codes_np, scales_np, global_scale, device="cuda"):
        codes = torch.from_numpy(codes_np).to(device)
        scales = torch.from_numpy(scales_np).to(device)
        gs = torch.tensor([float(global_scale)], dtype=torch.float32, device=device)
        return NVFP4Tensor(codes.shape[0], codes.shape[1] * 2, device, codes, scales, gs)


def nvfp4_workspace_bytes(op, a, b=0, c=0):
    return int(lib().nvfp4_workspace_bytes(op, a, b, c))


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _wrong_rank(x, rank):
    return AssertionError(f"expected a tensor of {rank} dimensions, got {x.dim()}")


def nvfp4_quantize(x, block_axis=0, global_scale_in=None, out=None, workspace=None, stream=None):
    """x: bf16 [R, C] device tensor with unit stride along C. Returns an NVFP4Tensor."""
    if stream is not None and (out is None or workspace is None) and _elsewhere(stream):
        return _on(stream, nvfp4_quantize, x, block_axis, global_scale_in, out, workspace)
    if out is None:
        try:
            R, C = x.shape
        except ValueError:
            raise _wrong_rank(x, 2) from None
        out = NVFP4Tensor(R, C, x.device) if block_axis == 0 else NVFP4Tensor(C, R, x.device)
    _check(_host().quantize(x, block_axis, global_scale_in, out, workspace, _stream(stream)))
    return out


def nvfp4_gemm(A, W, out_dtype=OUT_F32, Y=None, stream=None):
    if stream is not None and Y is None and _elsewhere(stream):
        return _on(stream, nvfp4_gemm, A, W, out_dtype, Y)
    if Y is None:
        Y = _host().output(A.codes, A.rows, W.rows, out_dtype != OUT_F32)
    _check(_host().gemm(A, W, out_dtype, Y, _stream(stream)))
    return Y


def nvfp4_gemm_scale_out(A, W, Y=None, scale_out=None, workspace=None, stream=None):
    """bf16 Y = A W^T together with the NVFP4 tensor scale of Y (one float on the device).  Returns (Y, scale_out)."""
    if stream is not None and (Y is None or scale_out is None or workspace is None) and _elsewhere(stream):
        return _on(stream, nvfp4_gemm_scale_out, A, W, Y, scale_out, workspace)
    if Y is None:
        Y = _host().output(A.codes, A.rows, W.rows, True)
    if scale_out is None:
        scale_out = torch.empty(1, dtype=torch.float32, device=A.codes.device)
    _check(_host().gemm_scale_out(A, W, Y, scale_out, workspace, _stream(stream)))
    return Y, scale_out


def nvfp4_lora_down(x, a, out=None, workspace=None, stream=None):
    """T = bf16(x a^T): x bf16 [M, K] (unit stride along K), a bf16 [128, K] contiguous."""
    if stream is not None and (out is None or workspace is None) and _elsewhere(stream):
        return _on(stream, nvfp4_lora_down, x, a, out, workspace)
    if out is None:
        try:
            M, _ = x.shape
        except ValueError:
            raise _wrong_rank(x, 2) from None
        out = _host().output(x, M, LORA_RANK, True)
    _check(_host().lora_down(x, a, out, workspace, _stream(stream)))
    return out


def nvfp4_gemm_lora(A, W, t, b, lora_scale, out_dtype=OUT_F32, Y=None, stream=None):
    """nvfp4_gemm(A, W) + lora_scale * t b^T, fused; t bf16 [M, 128], b bf16 [N, 128], both contiguous."""
    if stream is not None and Y is None and _elsewhere(stream):
        return _on(stream, nvfp4_gemm_lora, A, W, t, b, lora_scale, out_dtype, Y)
    if Y is None:
        Y = _host().output(A.codes, A.rows, W.rows, out_dtype != OUT_F32)
    _check(_host().gemm_lora(A, W, t, b, lora_scale, out_dtype, Y, _stream(stream)))
    return Y


def nvfp4_gemm_act_quant(A, W, act=ACT_GELU_TANH, global_scale_in=None, out=None, h_bf16=None,
                         workspace=None, stream=None):
    if stream is not None and (out is None or workspace is None) and _elsewhere(stream):
        return _on(stream, nvfp4_gemm_act_quant, A, W, act, global_scale_in, out, h_bf16, workspace)
    if out is None:
        out = NVFP4Tensor(A.rows, W.rows, A.codes.device)
    _check(_host().gemm_act_quant(A, W, act, global_scale_in, out, h_bf16, workspace, _stream(stream)))
    return out


def _heads_out(x):
    try:
        T, H, d = x.shape
    except ValueError:
        raise _wrong_rank(x, 3) from None
    return NVFP4Tensor(T * H, d, x.device)


def nvfp4_kv_quant(kv, out=None, workspace=None, stream=None):
    """kv: contiguous bf16 [T, H, d]."""
    if stream is not None and (out is None or workspace is None) and _elsewhere(stream):
        return _on(stream, nvfp4_kv_quant, kv, out, workspace)
    if out is None:
        out = _heads_out(kv)
    _check(_host().kv_quant(kv, out, workspace, _stream(stream)))
    return out


def nvfp4_kv_quant_noalloc(kv, out, stream=None):
    """kv: contiguous bf16 [T, H, d]; `out` must be given: this entry point (and this wrapper) allocates nothing."""
    _check(_host().kv_quant_noalloc(kv, out, _stream(stream)))
    return out


def nvfp4_quantize_4over6(x, global_scale_in=None, out=None, workspace=None, stream=None):
    """x: bf16 [R, C] device tensor with unit stride along C; blocks along C, scale search per block."""
    if stream is not None and (out is None or workspace is None) and _elsewhere(stream):
        return _on(stream, nvfp4_quantize_4over6, x, global_scale_in, out, workspace)
    if out is None:
        try:
            R, C = x.shape
        except ValueError:
            raise _wrong_rank(x, 2) from None
        out = NVFP4Tensor(R, C, x.device)
    _check(_host().quantize_4over6(x, global_scale_in, out, workspace, _stream(stream)))
    return out


def nvfp4_kv_quant_4over6(kv, out=None, workspace=None, stream=None):
    """kv: contiguous bf16 [T, H, d]; scale search per block."""
    if stream is not None and (out is None or workspace is None) and _elsewhere(stream):
        return _on(stream, nvfp4_kv_quant_4over6, kv, out, workspace)
    if out is None:
        out = _heads_out(kv)
    _check(_host().kv_quant_4over6(kv, out, workspace, _stream(stream)))
    return out


def nvfp4_quantize_for_all_to_all(x, P, global_scale_in=None, out=None, workspace=None, stream=None):
    """x: contiguous bf16 [T, H, d]; NVFP4 along d, rows regrouped into P per-destination slabs of H/P heads."""
    if stream is not None and (out is None or workspace is None) and _elsewhere(stream):
        return _on(stream, nvfp4_quantize_for_all_to_all, x, P, global_scale_in, out, workspace)
    if out is None:
        out = _heads_out(x)
    _check(_host().quantize_for_all_to_all(x, P, global_scale_in, out, workspace, _stream(stream)))
    return out


def nvfp4_quantize_rht(x, sign_mask, global_scale_in=None, out=None, workspace=None, stream=None):
    """x: bf16 [R, C], contracted over R.  Random Hadamard transform along R (groups of 16) with the
    16-bit sign mask, then the transposed quantizer: returns NVFP4Tensor [C, R]."""
    if stream is not None and (out is None or workspace is None) and _elsewhere(stream):
        return _on(stream, nvfp4_quantize_rht, x, sign_mask, global_scale_in, out, workspace)
    if out is None:
        try:
            R, C = x.shape
        except ValueError:
            raise _wrong_rank(x, 2) from None
        out = NVFP4Tensor(C, R, x.device)
    _check(_host().quantize_rht(x, int(sign_mask), global_scale_in, out, workspace, _stream(stream)))
    return out


def nvfp4_quantize_2d(w, global_scale_in=None, transposed=True, workspace=None, stream=None):
    """w: bf16 [R, C] weights (R, C multiples of 16), one scale per 16x16 tile.
    Returns (NVFP4Tensor [R, C], NVFP4Tensor [C, R] or None)."""
    if stream is not None and _elsewhere(stream):
        return _on(stream, nvfp4_quantize_2d, w, global_scale_in, transposed, workspace)
    try:
        R, C = w.shape
    except ValueError:
        raise _wrong_rank(w, 2) from None
    out = NVFP4Tensor(R, C, w.device)
    out_t = NVFP4Tensor(C, R, w.device) if transposed else None
    _check(_host().quantize_2d(w, global_scale_in, out, out_t, workspace, _stream(stream)))
    return out, out_t


def nvfp4_kv_quant_k(k, out=None, row_mean=None, workspace=None, stream=None):
    """k: contiguous bf16 [T, H, d] keys; K-smoothing then scale search.  Returns (NVFP4Tensor, row means bf16 [T*H])."""
    if stream is not None and (out is None or row_mean is None or workspace is None) and _elsewhere(stream):
        return _on(stream, nvfp4_kv_quant_k, k, out, row_mean, workspace)
    if out is None:
        out = _heads_out(k)
    if row_mean is None:
        try:
            T, H, _ = k.shape
        except ValueError:
            raise _wrong_rank(k, 3) from None
        row_mean = torch.empty(T * H, dtype=torch.bfloat16, device=k.device)
    _check(_host().kv_quant_k(k, out, row_mean, workspace, _stream(stream)))
    return out, row_mean


def nvfp4_kv_dequant_gather(chunks, H, d, out=None, stream=None):
    """chunks: list of (NVFP4Tensor, row_mean or None, T).  Returns bf16 [sum T, H, d]."""
    if stream is not None and out is None and _elsewhere(stream):
        return _on(stream, nvfp4_kv_dequant_gather, chunks, H, d, out)
    if out is None:
        out = torch.empty((sum(T for _, _, T in chunks), H, d), dtype=torch.bfloat16, device=chunks[0][0].codes.device)
    _check(_host().kv_dequant_gather(chunks, H, d, out, _stream(stream)))
    return out


def nvfp4_kv_dequant(q, T, H, d, out=None, stream=None):
    if stream is not None and out is None and _elsewhere(stream):
        return _on(stream, nvfp4_kv_dequant, q, T, H, d, out)
    if out is None:
        out = torch.empty((T, H, d), dtype=torch.bfloat16, device=q.codes.device)
    _check(_host().kv_dequant(q, T, H, d, out, _stream(stream)))
    return out


class NVFP4Rope:
    """Rotation of queries and keys: positions int32 [T, axes], freqs fp32 [pairs] (radians per position of each pair),
    axis_pairs the number of pairs that go by each axis, in order (one axis for text; time, height, width for video).
    interleaved: pairs of neighbours (2j, 2j + 1), else halves (j, j + pairs)."""

    def __init__(self, positions, freqs, axis_pairs, interleaved=True):
        self.positions, self.freqs = positions, freqs
        self.axis_pairs, self.interleaved = tuple(int(n) for n in axis_pairs), bool(interleaved)

    def _native(self):
        return self.positions, self.freqs, self.axis_pairs, self.interleaved


def nvfp4_qk_norm_rope(q, k, q_weight, k_weight, rope, eps=1e-6, q_out=None, k_out=None, stream=None):
    """q [T, Hq, d], k [T, Hk, d] bf16 (contiguous heads, any token stride; either may be None): RMS norm of each head with
    weights bf16 [d] (None: rotated only), then the rotation (an NVFP4Rope, or None).  q_out, k_out may be q and k.  Returns (q_out, k_out)."""
    if stream is not None and _elsewhere(stream):
        return _on(stream, nvfp4_qk_norm_rope, q, k, q_weight, k_weight, rope, eps, q_out, k_out)
    rc, q_out, k_out = _host().qk_norm_rope(q, k, q_weight, k_weight, rope and rope._native(), eps, q_out, k_out, _stream(stream))
    _check(rc)
    return q_out, k_out


def nvfp4_qk_norm_rope_backward(dq, dk, q, k, q_weight, k_weight, rope, eps=1e-6, dq_in=None, dk_in=None, dq_weight=None, dk_weight=None,
                                weight_grads=True, workspace=None, stream=None):
    """Gradients of nvfp4_qk_norm_rope from those of its outputs (dq, dk) and its inputs.  Returns (dq_in, dk_in, dq_weight,
    dk_weight): bf16 like dq and dk, and fp32 [d] (None without a weight, or with weight_grads=False)."""
    if stream is not None and _elsewhere(stream):
        return _on(stream, nvfp4_qk_norm_rope_backward, dq, dk, q, k, q_weight, k_weight, rope, eps, dq_in, dk_in, dq_weight, dk_weight, weight_grads, workspace)
    rc, dq_in, dk_in, dq_weight, dk_weight = _host().qk_norm_rope_backward(dq, dk, q, k, q_weight, k_weight, rope and rope._native(), eps, dq_in, dk_in,
                                                                           dq_weight, dk_weight, 1 if weight_grads else 0, workspace, _stream(stream))
    _check(rc)
    return dq_in, dk_in, dq_weight, dk_weight


class NVFP4KvCache:
    """Paged NVFP4 cache (see include/nvfp4.h): codes u8 [n_pages, page_tokens, H, d/2], scales u8 [n_pages, page_tokens, H, d/16],
    tensor scales fp32 [n_pages], and for smoothed keys the row means bf16 [n_pages, page_tokens, H]."""

    def __init__(self, k_codes, k_scales, k_global, v_codes, v_scales, v_global, k_mean=None):
        if k_codes.dim() != 4:
            raise _wrong_rank(k_codes, 4)
        n, p, H, half = k_codes.shape
        for name, t, shape, dtype in (("k_codes", k_codes, (n, p, H, half), torch.uint8), ("k_scales", k_scales, (n, p, H, half // 8), torch.uint8),
                                      ("k_global", k_global, (n,), torch.float32), ("v_codes", v_codes, (n, p, H, half), torch.uint8),
                                      ("v_scales", v_scales, (n, p, H, half // 8), torch.uint8), ("v_global", v_global, (n,), torch.float32),
                                      ("k_mean", k_mean, (n, p, H), torch.bfloat16)):
            if t is None and name == "k_mean":
                continue
            assert t.dtype == dtype and tuple(t.shape) == shape and t.is_contiguous(), f"{name}: expected a contiguous {dtype} tensor {shape}"
        self.k_codes, self.k_scales, self.k_global, self.k_mean = k_codes, k_scales, k_global, k_mean
        self.v_codes, self.v_scales, self.v_global = v_codes, v_scales, v_global
        self.n_pages, self.page_tokens, self.H, self.d = n, p, H, 2 * half
        self._native = (k_codes, k_scales, k_global, k_mean, v_codes, v_scales, v_global)

    @staticmethod
    def empty(n_pages, page_tokens, H, d, smooth=False, device="cuda"):
        """A cache without contents: codes and scales of zero, tensor scales of one."""
        planes = [torch.zeros((n_pages, page_tokens, H, w), dtype=torch.uint8, device=device) for w in (d // 2, d // 16) * 2]
        k_global, v_global = (torch.ones(n_pages, dtype=torch.float32, device=device) for _ in range(2))
        mean = torch.zeros((n_pages, page_tokens, H), dtype=torch.bfloat16, device=device) if smooth else None
        return NVFP4KvCache(planes[0], planes[1], k_global, planes[2], planes[3], v_global, mean)

    def page(self, i):
        """(keys, row means or None, values) of page i as NVFP4Tensors on the cache's memory: what the chunk quantizers take as `out`."""
        rows = self.page_tokens * self.H
        k = NVFP4Tensor(rows, self.d, None, self.k_codes[i].view(rows, -1), self.k_scales[i].view(rows, -1), self.k_global[i:i + 1])
        v = NVFP4Tensor(rows, self.d, None, self.v_codes[i].view(rows, -1), self.v_scales[i].view(rows, -1), self.v_global[i:i + 1])
        return k, None if self.k_mean is None else self.k_mean[i].view(rows), v


def nvfp4_kv_cache_write(cache, k, v, slots, scale_search=False, stream=None):
    """Quantizes k, v (bf16 [T, H, d], contiguous heads, any token stride; either may be None) into the slots (int64 [T]) of the cache."""
    if stream is not None and _elsewhere(stream):
        return _on(stream, nvfp4_kv_cache_write, cache, k, v, slots, scale_search)
    _check(_host().kv_cache_write(cache._native, k, v, slots, 1 if scale_search else 0, _stream(stream)))
    return cache


def nvfp4_kv_cache_read(cache, slots, k_out=None, v_out=None, stream=None):
    """Slots (int64 [T]) back to bf16 [T, H, d].  Returns (k_out, v_out); with one of the two given, the other is not read (None).
    Rows of slots outside the cache: zeros in new outputs, left as they were in given ones."""
    if stream is not None and _elsewhere(stream):
        return _on(stream, nvfp4_kv_cache_read, cache, slots, k_out, v_out)
    rc, k_out, v_out = _host().kv_cache_read(cache._native, slots, k_out, v_out, _stream(stream))
    _check(rc)
    return k_out, v_out


def nvfp4_kv_attention_workspace_bytes(total_q, Hq, H, d, max_kv, B, max_q, window=0, sink=0):
    return int(lib().nvfp4_kv_attention_workspace_bytes(total_q, Hq, H, d, max_kv, B, max_q, window, sink))


def nvfp4_kv_attention(q, cache, page_table, kv_lens, q_starts, max_q, softmax_scale=None, causal=False, window=0, sink=0, out_dtype=OUT_BF16,
                       out=None, lse=None, workspace=None, stream=None):
    """Attention of q (bf16 [total_q, Hq, d], contiguous heads, any token stride) over the cache: page_table int32 [B, max_pages],
    kv_lens int32 [B], q_starts int32 [B + 1]; softmax_scale d ** -0.5 by default.  Returns (out [total_q, Hq, d], lse fp32 [total_q, Hq]).
    Rows that no sequence computes (before the first query, behind the last one, from max_q on): zeros and -inf in new outputs, left as
    they were in given ones."""
    if stream is not None and _elsewhere(stream):
        return _on(stream, nvfp4_kv_attention, q, cache, page_table, kv_lens, q_starts, max_q, softmax_scale, causal, window, sink, out_dtype, out, lse, workspace)
    rc, out, lse = _host().kv_attention(q, cache._native, page_table, kv_lens, q_starts, max_q, cache.d ** -0.5 if softmax_scale is None else softmax_scale,
                                        1 if causal else 0, window, sink, out_dtype, out, lse, workspace, _stream(stream))
    _check(rc)
    return out, lse


def nvfp4_gemm_plan(M, N, K):
    """-> list of (tile, workgroups) per launch, e.g. [("256x256", 768), ("64x64", 192)]; host only."""
    buf = ctypes.create_string_buffer(256)
    _check(min(lib().nvfp4_gemm_plan(M, N, K, buf, len(buf)), 0))
    return [(item.split(":")[0], int(item.split(":")[1])) if ":" in item else (item, 0)
            for item in buf.value.decode().split()]


def nvfp4_set_timing(enabled):
    lib().nvfp4_set_timing(1 if enabled else 0)


def nvfp4_set_timing_ops(ops):
    """Record events only around the entry points listed in `ops` (OP_* ids); an empty list: none."""
    mask = 0
    for op in ops:
        mask |= 1 << op
    lib().nvfp4_set_timing_ops(mask)


def nvfp4_timing_read(op):
    """-> (calls, total_ms) recorded for entry point `op` since timing was enabled."""
    n, ms = ctypes.c_int(0), ctypes.c_float(0)
    _check(lib().nvfp4_timing_read(op, ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value


ONE_LAUNCH_AUTO, ONE_LAUNCH_ALWAYS, ONE_LAUNCH_NEVER = 0, 1, 2


def nvfp4_set_one_launch(mode=ONE_LAUNCH_AUTO):
    """Form of the row quantizers for tensors that fit on the chip (see include/nvfp4.h)."""
    _check(lib().nvfp4_set_one_launch(int(mode)))


def nvfp4_set_sync_spin_limit(ticks_10ns=0xFFFFFFFF):
    """Bound of the grid-wide wait of the one-launch quantizers (10 ns ticks; 0: give up at once; default: restore)."""
    lib().nvfp4_set_sync_spin_limit(ticks_10ns)


def nvfp4_timing_read_all(op, max_records=8192):
    """-> list of the recorded durations (ms) of entry point `op`, in call order."""
    buf = (ctypes.c_float * max_records)()
    n = lib().nvfp4_timing_read_all(op, buf, max_records)
    _check(min(n, 0))
    return [buf[i] for i in range(n)]


PROBE_READ, PROBE_WRITE, PROBE_COPY, PROBE_MFMA = 0, 1, 2, 3
PROBE_MFMA_FLOPS_PER_ITER = 256 * 4 * 64 * 32768


def nvfp4_probe(kind, a, b, nbytes=0, iters=0, stream=None):
    """Ceiling probe (see include/nvfp4.h): a, b device tensors (a may be None for write / mfma)."""
    _check(lib().nvfp4_probe(kind, _ptr(a), _ptr(b), int(nbytes), int(iters), _stream(stream)))


def bf16_from_bits(bits_np, device="cuda"):
    """uint16 numpy bit patterns -> bf16 device tensor (a copy, no arithmetic)."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(bits_np).view(np.int16)).to(device)
    return t.view(torch.bfloat16)


def bits_from_bf16(t):
    import numpy as np
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
