"""Argument checks of the norm / rotation, paged cache and attention entry points, and the attention plan: no GPU needed.
Pointers are fake but never dereferenced: validation fails first."""
import ctypes
import types

import pytest
import torch

import paper_2605_18739_amd as nv
from paper_2605_18739_amd.binding import _CHeads, _CHeadsGrad, _CKvCache, _CRope

NULL, SHAPE, ALIGN, WORKSPACE = -1, -2, -3, -4
P = 0x10000                                            # a 16-byte aligned address
NO_STREAM = types.SimpleNamespace(cuda_stream=0)


def ref(x):
    return None if x is None else ctypes.byref(x)


def heads(x=P, ld=512, weight=P, out=P, ld_out=512, H=4):
    return _CHeads(x, ld, weight, out, ld_out, H)


def rope(positions=P, freqs=P, axes=3, pairs=(22, 21, 21, 0), interleaved=1):
    return _CRope(positions, freqs, axes, (ctypes.c_int64 * 4)(*pairs), interleaved)


def norm(q, k=None, T=5, d=128, eps=1e-6, r=None):
    return nv.lib().nvfp4_qk_norm_rope(ref(q), ref(k), T, d, eps, ref(r), None)


def test_norm_rope_refuses():
    assert norm(None) == NULL
    assert norm(heads(x=None)) == NULL and norm(heads(out=None)) == NULL
    assert norm(heads(), heads(x=None)) == NULL
    assert norm(heads(), r=rope(positions=None)) == NULL and norm(heads(), r=rope(freqs=None)) == NULL
    for T in (0, -1, (1 << 30) + 1):
        assert norm(heads(), T=T) == SHAPE
    for d in (0, -16, 24, 272, 120):
        assert norm(heads(ld=4096, ld_out=4096), d=d) == SHAPE
    for H in (0, -1, 5):                               # (5 heads of 128 do not fit into 512)
        assert norm(heads(H=H)) == SHAPE
    assert norm(heads(ld=504)) == SHAPE and norm(heads(ld_out=0)) == SHAPE and norm(heads(ld=1 << 33)) == SHAPE
    assert norm(heads(H=1 << 20, ld=1 << 27, ld_out=1 << 27)) == SHAPE
    for eps in (0.0, -1e-6, float("nan"), float("inf"), 1e-42):
        assert norm(heads(), eps=eps) == SHAPE
    assert norm(heads(), r=rope(axes=5)) == SHAPE and norm(heads(), r=rope(axes=-1)) == SHAPE
    assert norm(heads(), r=rope(pairs=(22, 21, 22, 0))) == SHAPE                       # more than d / 2
    assert norm(heads(), r=rope(pairs=(22, -1, 21, 0))) == SHAPE
    assert norm(heads(), r=rope(pairs=(20, 20, 20, 0), interleaved=0)) == SHAPE        # halves: a multiple of eight
    assert norm(heads(), r=rope(pairs=(1 << 62, 1 << 62, 1 << 62, 0))) == SHAPE
    for h in (heads(x=P + 2), heads(out=P + 8), heads(weight=P + 4), heads(ld=516), heads(ld_out=524)):
        assert norm(h) == ALIGN
    assert norm(heads(), r=rope(positions=P + 2)) == ALIGN and norm(heads(), r=rope(freqs=P + 1)) == ALIGN


def grad(dy=P, ld_dy=512, x=P, ld_x=512, weight=P, dx=P, ld_dx=512, dweight=P, H=4):
    return _CHeadsGrad(dy, ld_dy, x, ld_x, weight, dx, ld_dx, dweight, H)


def backward(q, k=None, T=5, d=128, eps=1e-6, r=None, ws=P, n=1 << 30):
    return nv.lib().nvfp4_qk_norm_rope_backward(ref(q), ref(k), T, d, eps, ref(r), ws, n, None)


def test_norm_rope_backward_refuses():
    assert backward(None) == NULL
    for g in (grad(dy=None), grad(dx=None), grad(x=None)):
        assert backward(g) == NULL
    for g in (grad(ld_dy=504), grad(ld_x=504), grad(ld_dx=504), grad(H=5), grad(H=0)):
        assert backward(g) == SHAPE
    for g in (grad(dy=P + 2), grad(x=P + 2), grad(weight=P + 2), grad(dx=P + 2), grad(dweight=P + 2), grad(ld_dy=516), grad(ld_x=516), grad(ld_dx=516)):
        assert backward(g) == ALIGN
    need = nv.nvfp4_workspace_bytes(nv.OP_QK_NORM_ROPE_BACKWARD, 5, 128)
    assert need > 0 and nv.nvfp4_workspace_bytes(nv.OP_QK_NORM_ROPE_BACKWARD, 0, 128) == 0
    assert backward(grad(), ws=None) == WORKSPACE and backward(grad(), n=need - 1) == WORKSPACE and backward(grad(), ws=P + 4) == ALIGN
    assert backward(grad(), T=0) == SHAPE and backward(grad(), eps=0.0) == SHAPE


def cache(**kw):
    f = dict(k_codes=P, k_scales=P, k_global=P, k_mean=P, v_codes=P, v_scales=P, v_global=P, n_pages=10, page_tokens=32, H=4, d=128)
    f.update(kw)
    return _CKvCache(*(f[n] for n, _ in _CKvCache._fields_))


BAD_CACHES = [(dict([(n, None)]), NULL) for n in ("k_codes", "k_scales", "k_global", "v_codes", "v_scales", "v_global")] + [
    (dict(n_pages=0), SHAPE), (dict(n_pages=-1), SHAPE), (dict(n_pages=1 << 31), SHAPE), (dict(page_tokens=0), SHAPE), (dict(page_tokens=24), SHAPE),
    (dict(page_tokens=1 << 31), SHAPE), (dict(n_pages=1 << 30, page_tokens=1 << 20), SHAPE), (dict(H=0), SHAPE), (dict(H=1 << 22), SHAPE),
    (dict(d=0), SHAPE), (dict(d=72), SHAPE), (dict(d=288), SHAPE)] + [
    (dict([(n, P + 4)]), ALIGN) for n in ("k_codes", "k_scales", "v_codes", "v_scales")] + [(dict(k_global=P + 2), ALIGN), (dict(v_global=P + 1), ALIGN), (dict(k_mean=P + 2), ALIGN)]


def write(c, k=P, ldk=512, v=P, ldv=512, slots=P, T=3, search=0):
    return nv.lib().nvfp4_kv_cache_write(ref(c), k, ldk, v, ldv, slots, T, search, None)


def read(c, slots=P, T=3, k=P, v=P):
    return nv.lib().nvfp4_kv_cache_read(ref(c), slots, T, k, v, None)


def test_cache_write_and_read_refuse():
    for fields, status in BAD_CACHES:
        assert write(cache(**fields)) == status and read(cache(**fields)) == status, fields
    assert write(None) == NULL and read(None) == NULL
    assert write(cache(), k=None, v=None) == NULL and write(cache(), slots=None) == NULL
    assert read(cache(), k=None, v=None) == NULL and read(cache(), slots=None) == NULL
    for T in (0, -3, 1 << 30):
        assert write(cache(), T=T) == SHAPE and read(cache(), T=T) == SHAPE
    assert write(cache(), ldk=504) == SHAPE and write(cache(), ldv=0) == SHAPE
    assert write(cache(d=80, H=2)) == SHAPE                                             # smoothed keys: d / 16 a power of two
    assert write(cache(), k=P + 2) == ALIGN and write(cache(), v=P + 8) == ALIGN and write(cache(), ldk=516) == ALIGN and write(cache(), ldv=516) == ALIGN
    assert write(cache(), slots=P + 4) == ALIGN and read(cache(), slots=P + 4) == ALIGN
    assert read(cache(), k=P + 2) == ALIGN and read(cache(), v=P + 2) == ALIGN


def attention(c=None, **kw):
    f = dict(q=P, ldq=1024, total_q=7, Hq=8, table=P, max_pages=6, lens=P, starts=P, B=2, max_q=4, scale=0.1, causal=1, window=0, sink=0, out=P, ldo=1024,
             dtype=1, lse=P, ws=P, n=1 << 40)
    f.update(kw)
    return nv.lib().nvfp4_kv_attention(f["q"], f["ldq"], f["total_q"], f["Hq"], ref(c or cache()), f["table"], f["max_pages"], f["lens"], f["starts"], f["B"], f["max_q"],
                                       f["scale"], f["causal"], f["window"], f["sink"], f["out"], f["ldo"], f["dtype"], f["lse"], f["ws"], f["n"], None)


def test_attention_refuses():
    for fields, status in BAD_CACHES:
        assert attention(cache(**fields)) == status, fields
    for n in ("q", "table", "lens", "starts", "out"):
        assert attention(**{n: None}) == NULL, n
    for fields in (dict(total_q=0), dict(total_q=1 << 28), dict(Hq=6), dict(Hq=0), dict(B=0), dict(B=1 << 29), dict(max_q=0), dict(max_q=-1), dict(max_pages=0),
                   dict(max_pages=1 << 26), dict(ldq=1016), dict(ldo=1016), dict(window=-1), dict(sink=-1), dict(dtype=2), dict(scale=0.0), dict(scale=-1.0),
                   dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attention(**fields) == SHAPE, fields
    for fields in (dict(q=P + 2), dict(out=P + 8), dict(ldq=1028), dict(ldo=1028), dict(table=P + 2), dict(lens=P + 1), dict(starts=P + 2), dict(lse=P + 2), dict(ldo=1026, dtype=0)):
        assert attention(**fields) == ALIGN, fields
    need = nv.nvfp4_kv_attention_workspace_bytes(1, 8, 4, 128, 32 * 1000, 1, 1)
    big = dict(total_q=1, B=1, max_q=1, max_pages=1000)
    assert need > 0
    assert attention(**big, ws=None) == WORKSPACE and attention(**big, n=need - 1) == WORKSPACE and attention(**big, ws=P + 8) == ALIGN


def test_attention_workspace_covers_the_pieces():
    ws = nv.nvfp4_kv_attention_workspace_bytes
    assert ws(1, 8, 8, 128, 64, 1, 1) == 0                                              # one piece
    assert ws(1, 8, 8, 128, 1 << 20, 1, 1) % (8 * (128 * 4 + 8)) == 0
    assert ws(4, 8, 8, 128, 1 << 20, 4, 4000) == ws(4, 8, 8, 128, 1 << 20, 4, 4)        # no more queries than there are
    for bad in ((0, 8, 8, 128, 64, 1, 1), (1, 8, 3, 128, 64, 1, 1), (1, 8, 8, 120, 64, 1, 1), (1, 8, 8, 128, 0, 1, 1), (1, 8, 8, 128, 64, 0, 1), (1, 8, 8, 128, 64, 1, 0)):
        assert ws(*bad) == 0
    # a window bounds what is read, however long the cache
    assert ws(1, 8, 8, 128, 1 << 20, 1, 1, 100, 4) == ws(1, 8, 8, 128, 1 << 22, 1, 1, 100, 4) < ws(1, 8, 8, 128, 1 << 20, 1, 1)


def test_cache_handle_checks_its_tensors():
    c = nv.NVFP4KvCache.empty(3, 16, 2, 64, smooth=True, device="cpu")
    assert (c.n_pages, c.page_tokens, c.H, c.d) == (3, 16, 2, 64)
    k, mean, v = c.page(1)
    assert (k.rows, k.K) == (32, 64) and k.codes.data_ptr() == c.k_codes[1].data_ptr() and v.global_scale.data_ptr() == c.v_global[1:].data_ptr()
    assert mean.data_ptr() == c.k_mean[1].data_ptr()
    good = dict(k_codes=c.k_codes, k_scales=c.k_scales, k_global=c.k_global, v_codes=c.v_codes, v_scales=c.v_scales, v_global=c.v_global, k_mean=c.k_mean)
    nv.NVFP4KvCache(**good)
    for name in good:
        for wrong in (good[name].to(torch.float64), good[name][:2], good[name].unsqueeze(0)):
            with pytest.raises(AssertionError):
                nv.NVFP4KvCache(**{**good, name: wrong})
    with pytest.raises(AssertionError):
        nv.NVFP4KvCache(**{**good, "v_codes": c.v_codes.transpose(1, 2).contiguous().transpose(1, 2)})


def test_host_tensors_are_refused():
    c = nv.NVFP4KvCache.empty(3, 16, 2, 64, device="cpu")
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    w = torch.zeros(64, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    calls = [lambda: nv.nvfp4_qk_norm_rope(x, x, w, w, None, stream=NO_STREAM),
             lambda: nv.nvfp4_qk_norm_rope_backward(x, x, x, x, w, w, None, stream=NO_STREAM),
             lambda: nv.nvfp4_kv_cache_write(c, x, x, i.long(), stream=NO_STREAM),
             lambda: nv.nvfp4_kv_cache_read(c, i.long(), stream=NO_STREAM),
             lambda: nv.nvfp4_kv_attention(x, c, i.view(1, 4), i[:1], i[:2], 4, stream=NO_STREAM)]
    for call in calls:
        with pytest.raises((AssertionError, RuntimeError)):           # (RuntimeError: a machine without any GPU)
            call()


def test_attention_refuses_pages_past_its_addresses():
    assert attention(cache(n_pages=(1 << 30) + 1, page_tokens=16, H=1, d=16)) == SHAPE
    assert attention(cache(n_pages=1, page_tokens=1 << 28, H=2, d=128), max_pages=1, q=P + 2) == SHAPE      # 2^28 tokens of 2 x 8 scales
    assert attention(cache(n_pages=1, page_tokens=1 << 28, H=8, d=16), max_pages=1, q=P + 2) == SHAPE       # 2^28 tokens of 8 means
    assert attention(cache(n_pages=1, page_tokens=1 << 26, H=2, d=128), max_pages=1, Hq=8, q=P + 2) == ALIGN


def test_more_than_a_launch_covers_is_refused():
    """A launch has at most 2^32 - 1 lanes."""
    for T in (1 << 26, 1 << 30):
        assert norm(heads(), T=T) == SHAPE and backward(grad(), T=T) == SHAPE
    assert norm(heads(weight=P + 4), T=1 << 25) == ALIGN
    assert write(cache(), T=1 << 25) == SHAPE and read(cache(), T=1 << 25) == SHAPE        # two tensors, 32 blocks and 64 half blocks a row: a wave each
    assert write(cache(), T=1 << 24, slots=P + 4) == ALIGN
    ws = nv.nvfp4_kv_attention_workspace_bytes
    one = dict(Hq=8, max_q=1, max_pages=100)
    for B in (1 << 21, 1 << 26):                                                         # 2^24 rows of partial results and more
        assert attention(**one, total_q=B, B=B) == SHAPE and ws(B, 8, 4, 128, 3200, B, 1) == 0
    assert attention(**one, total_q=1 << 20, B=1 << 20, q=P + 2) == ALIGN and ws(1 << 20, 8, 4, 128, 3200, 1 << 20, 1) > 0
    many = dict(Hq=4, max_q=17, max_pages=1, total_q=1 << 27)                            # 17 rows of 4 heads: a workgroup each
    assert attention(**many, B=1 << 23) == SHAPE and ws(1 << 27, 4, 4, 128, 32, 1 << 23, 17) == 0
    assert attention(**many, B=1 << 20, q=P + 2) == ALIGN


def test_the_largest_window_is_as_good_as_none():
    ws = nv.nvfp4_kv_attention_workspace_bytes
    for total_q in (1, 300):
        none = ws(total_q, 8, 2, 128, 131072, 1, total_q)
        assert none > 0
        for window in (131072, 1 << 40, (1 << 63) - 1):
            for sink in (0, 1 << 40, (1 << 63) - 1):
                assert ws(total_q, 8, 2, 128, 131072, 1, total_q, window, sink) == none, (window, sink)


def test_attention_refuses_a_scale_that_leaves_the_range_as_a_power_of_two():
    for scale in (2.4e38, 3.4e38):
        assert attention(scale=scale) == SHAPE, scale
    assert attention(scale=2.3e38, q=P + 2) == ALIGN and attention(scale=1e-40, q=P + 2) == ALIGN


def test_flags_of_new_outputs_are_checked_like_the_calls_without():
    for flags in (0x100, 0x200, 0x300):
        assert attention(dtype=1 | flags, q=P + 2) == ALIGN and attention(dtype=flags, ldo=1026) == ALIGN and attention(dtype=2 | flags) == SHAPE
    assert attention(dtype=0x401) == SHAPE
    new = lambda c, slots=P, T=3, k=P, v=P: nv.lib().nvfp4_kv_cache_read_new(ref(c), slots, T, k, v, None)
    for fields, status in BAD_CACHES:
        assert new(cache(**fields)) == status, fields
    assert new(cache(), k=None, v=None) == NULL and new(cache(), T=0) == SHAPE and new(cache(), k=P + 2) == ALIGN


def test_short_caches_are_not_cut():
    """Up to 256 tokens (128 above d = 128) in one launch, 640 where the sequences are many."""
    ws = nv.nvfp4_kv_attention_workspace_bytes
    for d, tokens in ((64, 256), (128, 256), (144, 128), (256, 128)):
        for B in (1, 16):
            assert ws(B, 32, 8, d, tokens, B, 1) == 0 < ws(B, 32, 8, d, tokens + 32, B, 1), (d, B)
        assert ws(64, 32, 8, d, 640, 64, 1) == 0 < ws(64, 32, 8, d, 672, 64, 1), d
