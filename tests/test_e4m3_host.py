"""Argument checks of the 8-bit, gated and norm entry points: no GPU needed.  Pointers are fake but never dereferenced:
validation fails first."""
import ctypes

import pytest
import torch

import paper_2605_18739_amd as nv
from paper_2605_18739_amd.binding import _CE4m3Tensor

NULL, SHAPE, ALIGN, WORKSPACE = -1, -2, -3, -4
P = 0x10000                                            # a 16-byte aligned address
FAST = 0x400


def ref(x):
    return None if x is None else ctypes.byref(x)


def t8(rows=256, K=512, block_rows=1, codes=P, scales=P):
    return _CE4m3Tensor(codes, scales, rows, K, block_rows)


BAD_TENSORS = [(t8(codes=None), NULL), (t8(scales=None), NULL), (None, NULL), (t8(rows=0), SHAPE), (t8(rows=-1), SHAPE), (t8(rows=(1 << 30) + 1), SHAPE),
               (t8(K=0), SHAPE), (t8(K=24), SHAPE), (t8(K=(1 << 22) + 16), SHAPE), (t8(block_rows=0), SHAPE), (t8(block_rows=16), SHAPE),
               (t8(codes=P + 8), ALIGN), (t8(scales=P + 4), ALIGN)]


def quantize(out=None, x=P, R=256, C=512, ld=512, axis=0):
    return nv.lib().nvfp4_e4m3_quantize(x, R, C, ld, axis, ref(out), None)


def test_quantize_refuses():
    for t, status in BAD_TENSORS:
        assert quantize(t) == status
    ok = t8()
    assert quantize(ok, x=None) == NULL
    for bad in (dict(R=0), dict(C=0), dict(R=-4), dict(axis=2), dict(axis=-1), dict(C=520), dict(ld=504), dict(ld=(1 << 32) + 8), dict(R=255), dict(C=528)):
        assert quantize(ok, **bad) == SHAPE, bad
    assert quantize(t8(block_rows=128)) == SHAPE
    assert quantize(ok, x=P + 2) == ALIGN and quantize(ok, ld=516) == ALIGN
    # along the columns: the transpose, rows rounded up to sixteen
    assert quantize(t8(512, 256), R=255, axis=1, x=None) == NULL
    for t in (t8(512, 240), t8(512, 272), t8(256, 512), t8(512, 255)):
        assert quantize(t, R=255, axis=1) == SHAPE
    assert quantize(t8(516, 256), C=516, ld=520, axis=1) == SHAPE
    # more blocks than one launch covers
    assert quantize(t8(1 << 30, 1 << 22), R=1 << 30, C=1 << 22, ld=1 << 22) == SHAPE


def quantize_2d(out, out_t=None, w=P, R=256, C=512, ld=512):
    return nv.lib().nvfp4_e4m3_quantize_2d(w, R, C, ld, ref(out), ref(out_t), None)


def test_quantize_2d_refuses():
    ok = t8(block_rows=128)
    assert quantize_2d(None) == NULL and quantize_2d(ok, w=None) == NULL
    for bad in (dict(R=0), dict(C=-16), dict(R=255), dict(C=504), dict(ld=500), dict(R=240)):
        assert quantize_2d(ok, **bad) == SHAPE, bad
    assert quantize_2d(t8()) == SHAPE
    for t in (t8(512, 256), t8(256, 512, 128), t8(512, 272, 128)):
        assert quantize_2d(ok, t) == SHAPE
    assert quantize_2d(ok, t8(512, 256, 128, codes=None)) == NULL
    assert quantize_2d(ok, t8(512, 256, 128, codes=P + 4)) == ALIGN
    assert quantize_2d(ok, w=P + 8) == ALIGN and quantize_2d(ok, ld=516) == ALIGN


def gemm(A, W, Y=P, ldy=384, dtype=nv.OUT_F32):
    return nv.lib().nvfp4_e4m3_gemm(ref(A), ref(W), Y, ldy, dtype, None)


def test_gemm_refuses():
    A, W = t8(), t8(384, 512, 128)
    for t, status in BAD_TENSORS:
        assert gemm(t, W) == status and gemm(A, t) == status
    assert gemm(A, W, Y=None) == NULL
    assert gemm(A, t8(384, 528)) == SHAPE and gemm(t8(block_rows=128), W) == SHAPE
    for bad in (dict(ldy=383), dict(ldy=0), dict(ldy=-384), dict(ldy=(1 << 32) + 1), dict(dtype=2), dict(dtype=-1), dict(dtype=FAST | 2), dict(dtype=0x100)):
        assert gemm(A, W, **bad) == SHAPE, bad
    assert gemm(A, W, Y=P + 2) == ALIGN and gemm(A, W, Y=P + 1, dtype=nv.OUT_BF16) == ALIGN and gemm(A, W, Y=P + 2, dtype=FAST) == ALIGN
    # more tiles than one launch covers
    assert gemm(t8(1 << 30, 16), t8(1 << 30, 16), ldy=1 << 30) == SHAPE and gemm(t8(1, 16), t8(1 << 30, 16), ldy=1 << 30) == SHAPE


def gated(A, W, act=nv.ACT_SILU, out=None, h=None, ld_h=192, gu=None, ld_gu=384, ws=P, ws_bytes=1 << 30):
    return nv.lib().nvfp4_e4m3_gemm_gated(ref(A), ref(W), act, ref(out), h, ld_h, gu, ld_gu, ws, ws_bytes, None)


def test_gated_refuses():
    A, W, out = t8(), t8(384, 512, 128), t8(256, 192)
    for t, status in BAD_TENSORS:
        assert gated(t, W, out=out) == status and gated(A, t, out=out) == status
    assert gated(A, W) == NULL
    for act in (nv.ACT_NONE, 3, -1, FAST):
        assert gated(A, W, act=act, out=out) == SHAPE
    assert gated(A, t8(383, 512), out=out) == SHAPE and gated(A, t8(384, 528), out=out) == SHAPE
    for t in (t8(256, 208), t8(255, 192), t8(256, 192, 128)):
        assert gated(A, W, out=t) == SHAPE
    assert gated(A, t8(400, 512, 128), out=t8(256, 200)) == SHAPE                 # (F is no multiple of sixteen: no 8-bit result)
    assert gated(A, W, h=P, ld_h=191) == SHAPE and gated(A, W, gu=P, ld_gu=383) == SHAPE
    assert gated(A, W, h=P + 1) == ALIGN and gated(A, W, gu=P + 1) == ALIGN
    # up to 64 rows need a workspace for the 8-bit result
    few, out = t8(64), t8(64, 192)
    need = nv.nvfp4_workspace_bytes(nv.OP_E4M3_GEMM_GATED, 64, 192)
    assert need == 64 * 192 * 4 and nv.nvfp4_workspace_bytes(nv.OP_E4M3_GEMM_GATED, 65, 192) == 0 and nv.nvfp4_workspace_bytes(nv.OP_E4M3_GEMM_GATED, 0, 192) == 0
    assert gated(few, W, out=out, ws=None) == WORKSPACE and gated(few, W, out=out, ws_bytes=need - 1) == WORKSPACE and gated(few, W, out=out, ws=P + 8) == ALIGN


def backward(dh=P, ld_dh=256, gu=P, ld_gu=512, T=100, F=256, act=nv.ACT_SILU, out=None, out_t=None, h_t=None, d=None, ld_d=512):
    return nv.lib().nvfp4_gated_backward(dh, ld_dh, gu, ld_gu, T, F, act, ref(out), ref(out_t), ref(h_t), d, ld_d, None)


def test_gated_backward_refuses():
    out, out_t, h_t = t8(100, 512), t8(512, 112), t8(256, 112)
    assert backward() == NULL and backward(dh=None, out=out) == NULL and backward(gu=None, out=out) == NULL
    for bad in (dict(T=0), dict(F=0), dict(T=-1), dict(F=-128), dict(F=264), dict(act=nv.ACT_NONE), dict(act=5), dict(ld_dh=248), dict(ld_gu=504),
                dict(ld_dh=(1 << 22) + 8), dict(ld_gu=(1 << 22) + 8), dict(T=(1 << 22) + 1), dict(F=1 << 22)):
        assert backward(out=out, **bad) == SHAPE, bad
    assert backward(d=P, F=260, ld_dh=264, ld_gu=520, ld_d=520) == SHAPE
    assert backward(out=t8(100, 256)) == SHAPE and backward(out=t8(112, 512)) == SHAPE and backward(out=t8(100, 512, 128)) == SHAPE
    assert backward(out_t=t8(512, 96)) == SHAPE and backward(out_t=t8(256, 112)) == SHAPE and backward(h_t=t8(512, 112)) == SHAPE
    assert backward(out=out, out_t=out_t, h_t=t8(256, 112, codes=None)) == NULL
    assert backward(d=P, ld_d=504) == SHAPE and backward(d=P, ld_d=(1 << 22) + 8) == SHAPE
    assert backward(out=out, dh=P + 8) == ALIGN and backward(out=out, gu=P + 2) == ALIGN and backward(d=P + 8) == ALIGN
    assert backward(h_t=h_t, ld_dh=260) == ALIGN and backward(h_t=h_t, ld_gu=516) == ALIGN and backward(d=P, ld_d=516) == ALIGN


def norm(x=P, ld=512, r=None, ld_r=512, w=P, T=100, C=512, eps=1e-6, s=None, ld_s=512, out=None, y=None, ld_y=512):
    return nv.lib().nvfp4_rms_norm(x, ld, r, ld_r, w, T, C, eps, s, ld_s, ref(out), y, ld_y, None)


def test_rms_norm_refuses():
    out = t8(100, 512)
    assert norm() == NULL and norm(w=None, out=out) == NULL and norm(x=None, out=out) == NULL
    assert norm(r=P, out=out) == NULL and norm(s=P, out=out) == NULL              # a residual without a sum, a sum without a residual
    for bad in (dict(T=0), dict(C=0), dict(T=-1), dict(C=504), dict(C=16400, ld=16400), dict(T=1 << 30), dict(ld=504), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(eps=1e-42), dict(r=P, s=P, ld_r=500), dict(r=P, s=P, ld_s=500), dict(y=P, ld_y=100)):
        assert norm(out=out, **bad) == SHAPE, bad
    assert norm(out=t8(99, 512)) == SHAPE and norm(out=t8(100, 528)) == SHAPE and norm(out=t8(100, 512, 128)) == SHAPE
    for bad in (dict(x=P + 8), dict(w=P + 2), dict(y=P + 4), dict(ld=516), dict(y=P, ld_y=516), dict(r=P + 2, s=P), dict(r=P, s=P + 2), dict(r=P, s=P, ld_s=516)):
        assert norm(out=out, **bad) == ALIGN, bad


def norm_backward(dy=P, ld_dy=512, s=P, ld_s=512, w=P, ds=None, ld_ds=512, T=100, C=512, eps=1e-6, dx=P, ld_dx=512, dw=P, ws=P, ws_bytes=1 << 30):
    return nv.lib().nvfp4_rms_norm_backward(dy, ld_dy, s, ld_s, w, ds, ld_ds, T, C, eps, dx, ld_dx, dw, ws, ws_bytes, None)


def test_rms_norm_backward_refuses():
    for bad in (dict(dy=None), dict(s=None), dict(w=None), dict(dx=None)):
        assert norm_backward(**bad) == NULL, bad
    for bad in (dict(T=0), dict(C=24), dict(C=16400), dict(eps=0.0), dict(ld_dy=8), dict(ld_s=8), dict(ld_dx=8), dict(ds=P, ld_ds=8)):
        assert norm_backward(**bad) == SHAPE, bad
    for bad in (dict(dy=P + 2), dict(s=P + 2), dict(w=P + 2), dict(dx=P + 2), dict(ds=P + 2), dict(dw=P + 2), dict(ld_dy=516), dict(ws=P + 4)):
        assert norm_backward(**bad) == ALIGN, bad
    need = nv.nvfp4_workspace_bytes(nv.OP_RMS_NORM_BACKWARD, 100, 512)
    assert need == 100 * 512 * 4 and nv.nvfp4_workspace_bytes(nv.OP_RMS_NORM_BACKWARD, 1 << 20, 512) == 1024 * 512 * 4
    assert nv.nvfp4_workspace_bytes(nv.OP_RMS_NORM_BACKWARD, 0, 512) == 0 and nv.nvfp4_workspace_bytes(nv.OP_RMS_NORM_BACKWARD, 4, 16400) == 0
    assert norm_backward(ws=None) == WORKSPACE and norm_backward(ws_bytes=need - 1) == WORKSPACE


def test_tensor_checks():
    codes, scales = torch.zeros((256, 512), dtype=torch.float8_e4m3fn), torch.zeros((256, 4), dtype=torch.uint8).view(torch.float8_e8m0fnu)
    t = nv.E4M3Tensor(codes, scales)
    assert (t.rows, t.K, t.block_rows) == (256, 512, 1)
    t = nv.E4M3Tensor(codes.view(torch.uint8), scales[:2].view(torch.uint8))
    assert (t.rows, t.K, t.block_rows) == (256, 512, 128)
    for c, s in ((codes.float(), scales), (codes, scales.float()), (codes[:, ::2], scales), (codes, scales[:, :3]), (codes, scales[:3]), (codes[0], scales), (codes[:, :256], scales),
                 (codes, scales[::2]), (codes, scales[:, :3].contiguous())):
        with pytest.raises(AssertionError):
            nv.E4M3Tensor(c, s)
    with pytest.raises(AssertionError):
        nv.E4M3Tensor.empty(16, 16, block_rows=16, device="cpu")
    e = nv.E4M3Tensor.empty(300, 272, block_rows=128, device="cpu")
    assert tuple(e.scales.shape) == (3, 3) and e.codes.dtype == torch.float8_e4m3fn and e.scales.dtype == torch.float8_e8m0fnu
