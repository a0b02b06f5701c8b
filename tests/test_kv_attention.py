"""Norm and rotation of queries and keys, the paged NVFP4 cache and attention over it: GPU results against plain
evaluations in 64 bits.

Bounds (u = 2^-24, a half fp32 step; bf16 half step 2^-8, f16 2^-11, relative):
 norm/rotation  2^-8 |y| for the result's rounding, and 32 u (|a| + |b|) for the fp32 chain of a pair (a, b): the mean of
                squares (at most 14 rounded levels, halved by the root), root, two products, sine and cosine within 3 u, the
                turn's product and sum.
 gradients      the same with the sums of magnitudes that enter: dx 2^-8 |dx| + 64 u r (|w g| + |xh| mean |w g xh|);
                dweight (n + 64) u sum |g xh| over the n terms of a column.
 attention      2^-8 |o| (bf16) or 4 u |o| (fp32); the weights enter as f16, 2^-11 each of A = sum w |v| / sum w (two f16 numbers
                for fp32 output: 2^-22), and to 2^-25 of the largest, 2^-25 n max |v|; the scores' absolute error E = (d + 16) u
                (scale sum |q k| + 8) + 4 u |s| changes weights by a factor 1 + E, numerator and denominator: 2 E A;
                (n + 8) u A for the sums.
 lse            E + (n + 8) u + 4 u |lse|.
Codes, scale bytes, row means and reconstructed values: exact, against the oracle.
"""
import math

import numpy as np
import pytest
import torch

import paper_2605_18739_amd as nv
from paper_2605_18739_amd import workloads as wl
from tests.parity import dev_bf16

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def say(*a):
    print(*a, flush=True)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape):
    return torch.randn(shape, generator=g, dtype=F32)


# ---------------------------------------------------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------------------------------------------------
def split(pairs, axes):
    return [pairs - (axes - 1) * (pairs // axes)] + [pairs // axes] * (axes - 1) if axes else []


def rope_inputs(g, T, pairs, axes, far):
    parts = split(pairs, axes)
    positions = torch.randint(-far // 4, far, (T, axes), generator=g, dtype=torch.int32)
    freqs = torch.cat([10000.0 ** (-torch.arange(n, dtype=F64) / max(n, 1)) for n in parts] + [torch.empty(0, dtype=F64)]).to(F32)
    return positions, freqs, parts


def rotation(positions, freqs, parts, d, interleaved):
    """[T, d, d] rotations in 64 bits."""
    T, P = positions.shape[0], len(freqs)
    R = torch.eye(d, dtype=F64).repeat(T, 1, 1)
    axis = [x for x, n in enumerate(parts) for _ in range(n)]
    for j in range(P):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + P)
        angle = positions[:, axis[j]].double() * float(freqs[j])
        R[:, a, a] = R[:, b, b] = torch.cos(angle)
        R[:, a, b], R[:, b, a] = -torch.sin(angle), torch.sin(angle)
    return R


def norm_ref(x, w, R, eps):
    x = x.double()
    y = x if w is None else x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w.double()
    return torch.einsum("tab,thb->tha", R, y), torch.einsum("tab,thb->tha", R.abs(), y.abs())


def backward_ref(dy, x, w, R, eps):
    g = torch.einsum("tba,thb->tha", R, dy.double())
    ga = torch.einsum("tba,thb->tha", R.abs(), dy.double().abs())
    if w is None:
        return g, ga, None, None
    x, w = x.double(), w.double()
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    xh = x * r
    m = (w * g * xh).mean(-1, keepdim=True)
    dx = r * (w * g - xh * m)
    bound = r * ((w * ga).abs() + xh.abs() * (w * ga * xh).abs().mean(-1, keepdim=True))
    return dx, bound, (g * xh).sum((0, 1)), (ga * xh.abs()).sum((0, 1))


NORM_CASES = [
    # T, Hq, Hk, d, axes, pairs, interleaved, far, what
    (1, 1, 0, 16, 1, 8, True, 100, "one row of one block"),
    (1, 3, 1, 128, 1, 64, False, 2 ** 20, "a single token, far"),
    (7, 5, 2, 64, 2, 32, True, 1000, "two axes"),
    (13, 24, 24, 128, 3, 64, True, 64, "three axes, 22 + 21 + 21"),
    (9, 3, 3, 80, 1, 40, False, 4096, "head of 80, halves"),
    (6, 2, 5, 256, 4, 128, False, 300, "four axes, head of 256"),
    (5, 9, 1, 256, 3, 40, True, 300, "a third of the head turned"),
    (5, 4, 4, 96, 1, 16, False, 300, "32 of 96 turned"),
    (4, 7, 0, 48, 0, 0, True, 1, "norm alone, queries alone"),
    (1200, 2, 1, 32, 1, 16, True, 5000, "many tokens of few heads"),
    (4500, 1, 2, 16, 1, 8, False, 5000, "more tokens than waves"),
]


def norm_tensors(case, seed):
    T, Hq, Hk, d, axes, pairs, interleaved, far, what = case
    g = gen(seed)
    positions, freqs, parts = rope_inputs(g, T, pairs, axes, far)
    q, k = (randn(g, T, Hq, d) * torch.exp(randn(g, d))).to(BF), (randn(g, T, Hk, d) * 3).to(BF)
    if T > 3:
        q[2] = 0
    wq, wk = (1 + 0.3 * randn(g, d)).to(BF), (1 + 0.3 * randn(g, d)).to(BF)
    rope = nv.NVFP4Rope(positions.cuda(), freqs.cuda(), parts, interleaved) if pairs else None
    return g, q, k if Hk else None, wq, wk, rope, rotation(positions, freqs, parts, d, interleaved)


def cuda(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("case", NORM_CASES, ids=[c[-1] for c in NORM_CASES])
@pytest.mark.parametrize("normed", [True, False])
def test_norm_rope(case, normed):
    g, q, k, wq, wk, rope, R = norm_tensors(case, 11)
    eps = 1e-6
    if not normed:
        wq = None                                        # the keys keep theirs
    say("[norm_rope]", case[-1], normed)
    got = nv.nvfp4_qk_norm_rope(cuda(q), cuda(k), cuda(wq), cuda(wk), rope, eps=eps)
    torch.cuda.synchronize()
    for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
        if x is None:
            assert y is None
            continue
        want, pair = norm_ref(x, w, R, eps)
        err = (y.cpu().double() - want).abs()
        assert (err <= 2.0 ** -8 * want.abs() + 32 * U * pair + 1e-38).all(), float((err / (want.abs() + 1e-30)).max())


@pytest.mark.parametrize("case", NORM_CASES, ids=[c[-1] for c in NORM_CASES])
@pytest.mark.parametrize("normed", [True, False])
def test_norm_rope_backward(case, normed):
    g, q, k, wq, wk, rope, R = norm_tensors(case, 12)
    eps = 1e-6
    if not normed:
        wq = None
    dq, dk = (1e-2 * randn(g, *q.shape)).to(BF), None if k is None else (1e-2 * randn(g, *k.shape)).to(BF)
    say("[norm_rope_backward]", case[-1], normed)
    got = nv.nvfp4_qk_norm_rope_backward(cuda(dq), cuda(dk), cuda(q), cuda(k), cuda(wq), cuda(wk), rope, eps=eps)
    again = nv.nvfp4_qk_norm_rope_backward(cuda(dq), cuda(dk), cuda(q), cuda(k), cuda(wq), cuda(wk), rope, eps=eps)
    torch.cuda.synchronize()
    for a, b in zip(got, again):
        assert (a is None and b is None) or torch.equal(a, b)
    for x, dy, w, dx, dw in ((q, dq, wq, got[0], got[2]), (k, dk, wk, got[1], got[3])):
        if x is None:
            assert dx is None and dw is None
            continue
        want, bound, want_w, sum_w = backward_ref(dy, x, w, R, eps)
        err = (dx.cpu().double() - want).abs()
        assert (err <= 2.0 ** -8 * want.abs() + 64 * U * bound + 1e-38).all()
        if w is None:
            assert dw is None
        else:
            n = x.shape[0] * x.shape[1]
            assert ((dw.cpu().double() - want_w).abs() <= (n + 64) * U * sum_w + 1e-38).all()


def test_norm_rope_gradients_against_differences():
    """Central differences of the 64-bit forward pass, the upstream gradient a vector: what the kernel's gradients predict."""
    case = (3, 2, 1, 64, 2, 24, True, 50, "")
    g, q, k, wq, wk, rope, R = norm_tensors(case, 13)
    dq = (randn(g, *q.shape)).to(BF)
    dx, _, dw, _ = nv.nvfp4_qk_norm_rope_backward(cuda(dq), None, cuda(q), None, cuda(wq), None, rope)
    L = lambda x, w: float((norm_ref(x, w, R, 1e-6)[0] * dq.double()).sum())
    for seed in range(4):
        v = torch.randn(q.shape, generator=gen(seed), dtype=F64)
        h = 1e-5
        diff = (L(q.double() + h * v, wq) - L(q.double() - h * v, wq)) / (2 * h)
        slope = float((dx.cpu().double() * v).sum())
        assert abs(diff - slope) <= 2.0 ** -8 * float((dx.cpu().double() * v).abs().sum()) + 1e-4
        v = torch.randn(wq.shape, generator=gen(seed), dtype=F64)
        diff = (L(q, wq.double() + h * v) - L(q, wq.double() - h * v)) / (2 * h)
        assert abs(diff - float((dw.cpu().double() * v).sum())) <= 1e-4 * float(dw.abs().sum().cpu())


def test_norm_rope_inside_a_fused_projection_and_in_place():
    T, Hq, Hk, d = 21, 6, 2, 128
    g = gen(5)
    x = randn(g, T, (Hq + 2 * Hk) * d + 24).to(BF).cuda()
    q, k = x[:, :Hq * d].unflatten(1, (Hq, d)), x[:, Hq * d:(Hq + Hk) * d].unflatten(1, (Hk, d))
    positions, freqs, parts = rope_inputs(g, T, 64, 3, 90)
    w = (1 + 0.1 * randn(g, d)).to(BF).cuda()
    for interleaved in (True, False):
        rope = nv.NVFP4Rope(positions.cuda(), freqs.cuda(), parts, interleaved)
        want = nv.nvfp4_qk_norm_rope(q.contiguous(), k.contiguous(), w, w, rope)
        y = x.clone()
        yq, yk = y[:, :Hq * d].unflatten(1, (Hq, d)), y[:, Hq * d:(Hq + Hk) * d].unflatten(1, (Hk, d))
        a, b = nv.nvfp4_qk_norm_rope(yq, yk, w, w, rope, q_out=yq, k_out=yk)
        assert a is yq and torch.equal(a, want[0]) and torch.equal(b, want[1])
        assert torch.equal(y[:, (Hq + Hk) * d:], x[:, (Hq + Hk) * d:])                   # the values and the padding stay
        dq = randn(g, T, Hq, d).to(BF).cuda()
        want = nv.nvfp4_qk_norm_rope_backward(dq, None, q.contiguous(), None, w, None, rope)
        y = x.clone()
        yq = y[:, :Hq * d].unflatten(1, (Hq, d))
        got = nv.nvfp4_qk_norm_rope_backward(dq, None, yq, None, w, None, rope, dq_in=yq)       # the gradient over its input
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
        inplace = dq.clone()
        got = nv.nvfp4_qk_norm_rope_backward(inplace, None, q, None, w, None, rope, dq_in=inplace, weight_grads=False)
        assert torch.equal(got[0], want[0]) and got[2] is None


# ---------------------------------------------------------------------------------------------------------------------
# the cache
# ---------------------------------------------------------------------------------------------------------------------
def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def new_cache(pages, page, H, d, smooth, seed, amax=12.0):
    c = nv.NVFP4KvCache.empty(pages, page, H, d, smooth)
    for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales):
        t.fill_(0xEE)
    g = gen(seed)
    c.k_global.copy_(amax / 2688 * (0.5 + torch.rand(pages, generator=g)))
    c.v_global.copy_(amax / 2688 * (0.5 + torch.rand(pages, generator=g)))
    if smooth:
        c.k_mean.fill_(-77.0)
    return c


def check_slots(oracle, c, k, v, slots, search, what):
    """Every written slot holds the oracle's bytes; every other byte is as it was (0xEE)."""
    page = c.page_tokens
    written = torch.zeros(c.n_pages * page, dtype=torch.bool)
    slots = slots.cpu()
    ok = (slots >= 0) & (slots < c.n_pages * page)
    written[slots[ok]] = True
    for x, codes, scales, gs, mean in ((k, c.k_codes, c.k_scales, c.k_global, c.k_mean), (v, c.v_codes, c.v_scales, c.v_global, None)):
        codes, scales = codes.cpu().flatten(0, 1), scales.cpu().flatten(0, 1)
        untouched = ~written if x is not None else torch.ones_like(written)
        assert (codes[untouched] == 0xEE).all() and (scales[untouched] == 0xEE).all(), what
        if x is None:
            continue
        xb = bits(x)
        for p in range(c.n_pages):
            t = torch.nonzero(ok & (slots // page == p)).flatten()
            if len(t) == 0:
                continue
            rows = xb[t.numpy()].reshape(-1, c.d)
            if mean is not None:
                mu, rows = oracle.kv_smooth(rows)
                assert (bits(mean.flatten(0, 1)[slots[t]]).reshape(-1) == mu).all(), f"{what}: means"
            q = oracle.quantize(rows, global_scale_in=float(gs[p]), four_over_six=search)
            assert (scales[slots[t]].reshape(len(rows), -1).numpy() == q.scales).all(), f"{what}: scales of page {p}"
            assert (codes[slots[t]].reshape(len(rows), -1).numpy() == q.codes).all(), f"{what}: codes of page {p}"


CACHE_CASES = [
    # T, H, d, page, pages
    (1, 1, 16, 16, 1), (5, 1, 128, 16, 4), (33, 3, 80, 32, 3), (70, 8, 128, 48, 2), (19, 2, 256, 16, 5), (130, 24, 128, 80, 3), (9, 5, 64, 16, 2),
]


@pytest.mark.parametrize("case", CACHE_CASES)
@pytest.mark.parametrize("search", [False, True])
@pytest.mark.parametrize("smooth", [False, True])
def test_cache_write_and_read(oracle, case, search, smooth):
    T, H, d, page, pages = case
    if smooth and d == 80:
        pytest.skip("smoothed keys need d / 16 to be a power of two")
    say("[cache]", case, search, smooth)
    g = gen(T)
    c = new_cache(pages, page, H, d, smooth, 3)
    # rows of a fused projection; a token beyond the page's scale (saturated block scales), a row of zeros
    fused = (randn(g, T, 3 * H * d) * torch.exp(randn(g, T, 1))).to(BF)
    fused[T // 2] *= 40
    fused[T - 1, :d] = 0
    fused = fused.cuda()
    k, v = fused[:, H * d:2 * H * d].unflatten(1, (H, d)), fused[:, 2 * H * d:].unflatten(1, (H, d))
    slots = torch.randperm(pages * page, generator=g)[:T]
    slots = torch.cat([slots, torch.full((max(0, T - len(slots)),), -1)])
    if T > 4:
        slots[1], slots[3] = -5, pages * page                    # skipped
    dev = slots.to(torch.int64).cuda()
    nv.nvfp4_kv_cache_write(c, k, v, dev, scale_search=search)
    check_slots(oracle, c, k, v, slots, search, "written")
    # read back: exact reconstruction, rows of skipped slots as they were
    ko, vo = (torch.full((T, H, d), 5.0, dtype=BF, device="cuda") for _ in range(2))
    nv.nvfp4_kv_cache_read(c, dev, ko, vo)
    for out, codes, scales, gs, mean in ((ko, c.k_codes, c.k_scales, c.k_global, c.k_mean), (vo, c.v_codes, c.v_scales, c.v_global, None)):
        codes, scales = codes.flatten(0, 1).cpu().numpy(), scales.flatten(0, 1).cpu().numpy()
        for t, s in enumerate(slots.tolist()):
            if not 0 <= s < pages * page:
                assert (out[t] == 5.0).all()
                continue
            q = type("Q", (), {"codes": codes[s], "scales": scales[s], "global_scale": np.float32(float(gs[s // page])), "rows": H, "K": d})
            want = oracle.dequant_bf16(q, None if mean is None else bits(mean.flatten(0, 1)[s]))
            assert (bits(out[t]) == want).all(), (t, s)
    one = nv.nvfp4_kv_cache_read(c, dev, k_out=torch.full_like(ko, 5.0))
    assert one[1] is None and torch.equal(one[0], ko)


def test_cache_write_of_keys_alone_and_of_values_alone(oracle):
    T, H, d, page, pages = 40, 3, 64, 32, 3
    g = gen(9)
    k, v = randn(g, T, H, d).to(BF).cuda(), randn(g, T, H, d).to(BF).cuda()
    slots = torch.randperm(pages * page, generator=g)[:T]
    c = new_cache(pages, page, H, d, True, 4)
    nv.nvfp4_kv_cache_write(c, k, None, slots.cuda())
    check_slots(oracle, c, k, None, slots, False, "keys alone")
    c = new_cache(pages, page, H, d, True, 4)
    nv.nvfp4_kv_cache_write(c, None, v, slots.cuda(), scale_search=True)
    check_slots(oracle, c, None, v, slots, True, "values alone")
    assert (c.k_mean == -77.0).all()


def test_cache_scales_on_ties_and_outside_the_fp32_safe_range(oracle):
    """Page scales that are powers of two (quotients on midpoints) and far outside [2^-100, 2^100]."""
    H, d, page = 2, 64, 16
    g = np.random.default_rng(7)
    scales = [2.0 ** -9, 2.0 ** -7, 1e-33, 1e33, 21 / 2688, 3.0e-5]
    c = new_cache(len(scales), page, H, d, False, 1)
    c.k_global.copy_(torch.tensor(scales))
    c.v_global.copy_(torch.tensor(scales[::-1]))
    x = g.integers(-40, 41, size=(page * len(scales), H, d)).astype(np.float32) * np.float32(0.125)
    gain = np.repeat(np.array(scales, np.float32) * 512, page)[:, None, None]
    k = dev_bf16(wl.to_bf16_bits((x * gain).reshape(-1, H * d))).view(-1, H, d)
    v = dev_bf16(wl.to_bf16_bits((x * gain[::-1]).reshape(-1, H * d))).view(-1, H, d)
    slots = torch.arange(page * len(scales))
    for search in (False, True):
        c.k_codes.fill_(0xEE), c.v_codes.fill_(0xEE)
        nv.nvfp4_kv_cache_write(c, k, v, slots.cuda(), scale_search=search)
        check_slots(oracle, c, k, v, slots, search, "scales")


def test_a_page_is_what_the_chunk_quantizers_fill(oracle):
    """A page filled by nvfp4_kv_quant_k / nvfp4_kv_quant_4over6 reads back as nvfp4_kv_dequant_gather gives it, and a page
    written slot by slot with the same tensor scale holds the same bytes."""
    H, d, page = 3, 128, 48
    kb, vb = wl.kv_tensor(page, H, d, 3, 0), wl.kv_tensor(page, H, d, 3, 1)
    c = new_cache(3, page, H, d, True, 2)
    k, mean, v = c.page(1)
    nv.nvfp4_kv_quant_k(dev_bf16(kb), out=k, row_mean=mean)
    nv.nvfp4_kv_quant_4over6(dev_bf16(vb), out=v)
    slots = torch.arange(page, 2 * page, device="cuda")
    ko, vo = nv.nvfp4_kv_cache_read(c, slots)
    assert torch.equal(ko, nv.nvfp4_kv_dequant_gather([(k, mean, page)], H, d))
    assert torch.equal(vo.view(torch.int16), nv.nvfp4_kv_dequant(v, page, H, d).view(torch.int16))
    c2 = new_cache(3, page, H, d, True, 2)
    c2.k_global.copy_(c.k_global), c2.v_global.copy_(c.v_global)
    nv.nvfp4_kv_cache_write(c2, dev_bf16(kb), dev_bf16(vb), slots, scale_search=True)
    for a, b in zip(c._native, c2._native):
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------------
MAG = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=F64)
E4M3 = torch.tensor([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)], dtype=F64)


def held(codes, scales, gs, mean, page, slots):
    """Exact values [n, H, d] of the slots (on the cache's device)."""
    mag, e4m3 = MAG.to(codes.device), E4M3.to(codes.device)
    p = slots // page
    c, s = codes.flatten(0, 1)[slots].long(), scales.flatten(0, 1)[slots].long()
    both = torch.stack([c & 15, c >> 4], -1).flatten(-2)
    x = torch.where(both >= 8, -1.0, 1.0).double() * mag[both & 7]
    x = x * e4m3[s & 127].repeat_interleave(16, -1) * gs.double()[p].view(-1, 1, 1)
    return x if mean is None else x + mean.flatten(0, 1)[slots].double().unsqueeze(-1)


def fill_cache(c, g, k_gain=1.0):
    """Random codes, scale bytes around 1 (every code and sign, some blocks of zeros), means."""
    for codes, scales in ((c.k_codes, c.k_scales), (c.v_codes, c.v_scales)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8))
        scales.copy_(torch.randint(40, 80, scales.shape, generator=g, dtype=torch.uint8))
        scales.flatten()[::7] = 0
        scales.flatten()[::11] = 3                                 # subnormal
    c.k_global.copy_(k_gain * (0.5 + torch.rand(c.n_pages, generator=g)))
    c.v_global.copy_(torch.exp(2 * randn(g, c.n_pages)))           # pages whose values differ by orders of magnitude
    if c.k_mean is not None:
        c.k_mean.copy_((k_gain * randn(g, *c.k_mean.shape)).to(BF))


def attention_ref(q, c, table, lens, starts, max_q, scale, causal, window, sink, out_f32):
    """(out, lse, bound of out, bound of lse) in 64 bits; NaN in rows that no sequence computes."""
    total, Hq, d = q.shape
    G, page = Hq // c.H, c.page_tokens
    out, lse = torch.full((total, Hq, d), math.nan, dtype=F64), torch.full((total, Hq), math.nan, dtype=F64)
    bo, bl = torch.zeros_like(out), torch.zeros_like(lse)
    planes = [None if t is None else t.cpu() for t in c._native]
    for b in range(len(lens)):
        n, i0, nq = min(lens[b], table.shape[1] * page), starts[b], starts[b + 1] - starts[b]
        rows = min(nq, max_q)
        if rows <= 0:
            continue
        j = torch.arange(n)
        pages = table[b].long()[j // page]
        real = (pages >= 0) & (pages < c.n_pages)
        slots = pages.clamp(0, c.n_pages - 1) * page + j % page
        k = held(planes[0], planes[1], planes[2], planes[3], page, slots)
        v = held(planes[4], planes[5], planes[6], None, page, slots)
        p = n - nq + torch.arange(rows) if causal else torch.full((rows,), n - 1)
        see = (j[None] <= p[:, None]) & real[None]
        if window:
            see &= (j[None] > p[:, None] - window) | (j[None] < sink)
        for h in range(Hq):
            qh = q[i0:i0 + rows, h].cpu().double()
            s = (qh @ k[:, h // G].T * scale).masked_fill(~see, -math.inf)
            sa = qh.abs() @ k[:, h // G].abs().T * scale
            top = s.amax(-1, keepdim=True).clamp(min=-1e300) if n else torch.zeros(rows, 1, dtype=F64)
            w = torch.exp(s - top)
            total_w = w.sum(-1, keepdim=True)
            some = total_w > 0
            o = torch.where(some, w @ v[:, h // G] / total_w.clamp(min=1e-300), 0.0)
            A = torch.where(some, w @ v[:, h // G].abs() / total_w.clamp(min=1e-300), 0.0)
            E = ((d + 16) * U * (sa + 8) + 4 * U * s.abs()).masked_fill(~see, 0.0).amax(-1, keepdim=True) if n else torch.zeros(rows, 1, dtype=F64)
            vmax = torch.where(see.unsqueeze(-1), v[:, h // G].abs().unsqueeze(0), 0.0).amax((1, 2)).unsqueeze(-1) if n else torch.zeros(rows, 1, dtype=F64)
            out[i0:i0 + rows, h] = o
            bo[i0:i0 + rows, h] = ((4 * U if out_f32 else 2.0 ** -8) * o.abs() + ((2.0 ** -22 if out_f32 else 2.0 ** -11) + 2 * E + (n + 8) * U) * A
                                   + 2.0 ** -25 * n * vmax)
            lse[i0:i0 + rows, h] = (top + torch.log(total_w)).squeeze(-1)
            bl[i0:i0 + rows, h] = (E + (n + 8) * U).squeeze(-1) + 4 * U * torch.where(some, top.abs() + torch.log(total_w.clamp(min=1e-300)).abs(), 0.0).squeeze(-1)
    return out, lse, bo, bl


def attention_case(seed, lens, queries, Hq, H, d, page, smooth, extra_pages=2, gain=1.0):
    g = gen(seed)
    need = [-(-n // page) for n in lens]
    most, pages = max(max(need), 1), sum(need) + extra_pages
    c = new_cache(pages, page, H, d, smooth, seed)
    fill_cache(c, g, gain / math.sqrt(d))
    order = torch.randperm(pages, generator=g)
    table, at = torch.full((len(lens), most), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n].to(torch.int32)
        at += n
    starts = [sum(queries[:b]) for b in range(len(queries) + 1)]
    q = randn(g, starts[-1] + 2, Hq, d).to(BF)                      # two rows behind the last sequence
    return c, table, starts, q


def run_attention(c, table, lens, starts, q, max_q, causal, window=0, sink=0, out_f32=False, scale=None, check=True, **kw):
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    out = torch.full(q.shape, 3.0, dtype=F32 if out_f32 else BF, device="cuda")
    lse = torch.full(q.shape[:2], 4.0, dtype=F32, device="cuda")
    nv.nvfp4_kv_attention(q.cuda(), c, table.cuda(), dev(lens), dev(starts), max_q, softmax_scale=scale, causal=causal, window=window, sink=sink,
                          out_dtype=nv.OUT_F32 if out_f32 else nv.OUT_BF16, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    if check:
        want, want_lse, bo, bl = attention_ref(q, c, table, lens, starts, max_q, c.d ** -0.5 if scale is None else scale, causal, window, sink, out_f32)
        computed = ~torch.isnan(want)
        o, e = out.cpu().double(), lse.cpu().double()
        assert (o[~computed] == 3.0).all() and (e[torch.isnan(want_lse)] == 4.0).all(), "rows that no sequence owns"
        err = (o - want).abs()[computed]
        assert (err <= bo[computed]).all(), ("out", float((err / bo[computed].clamp(min=1e-300)).max()))
        rows = ~torch.isnan(want_lse)
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(e) & (e < 0), empty) and (o[empty] == 0).all(), "rows that see nothing"
        err = (e - want_lse).abs()[rows & ~empty]
        assert (err <= bl[rows & ~empty]).all(), ("lse", float((err / bl[rows & ~empty]).max()))
    return out, lse


DECODE = [
    # lens, Hq, H, d, page, smooth, what
    ([1], 1, 1, 64, 16, False, "one token"),
    ([0, 5, 16, 17, 33], 4, 4, 64, 16, False, "empty, inside and across pages"),
    ([700, 0, 129, 1024], 24, 24, 128, 48, True, "24 heads, smoothed"),
    ([300, 77], 32, 4, 128, 32, True, "eight heads to one"),
    ([513], 14, 2, 128, 16, False, "seven heads to one"),
    ([90, 200], 6, 3, 80, 16, False, "head of 80"),
    ([90, 200], 16, 16, 16, 32, True, "head of 16"),
    ([40, 1500], 3, 1, 256, 80, True, "head of 256"),
    ([333], 2, 2, 176, 16, False, "head of 176"),
    ([6000], 4, 1, 128, 64, False, "split over many waves"),
]


@pytest.mark.parametrize("case", DECODE, ids=[c[-1] for c in DECODE])
@pytest.mark.parametrize("out_f32", [False, True])
def test_attention_of_single_tokens(case, out_f32):
    lens, Hq, H, d, page, smooth, what = case
    say("[attention] decode", what, out_f32)
    c, table, starts, q = attention_case(21, lens, [1] * len(lens), Hq, H, d, page, smooth, gain=2.0)
    run_attention(c, table, lens, starts, q, 1, True, out_f32=out_f32)


@pytest.mark.parametrize("case", DECODE[1:], ids=[c[-1] for c in DECODE[1:]])
@pytest.mark.parametrize("window,sink", [(16, 0), (33, 5), (200, 40), (10 ** 12, 10 ** 12)])
def test_attention_of_single_tokens_in_a_window(case, window, sink):
    lens, Hq, H, d, page, smooth, what = case
    say("[attention] decode window", what, window, sink)
    c, table, starts, q = attention_case(22, lens, [1] * len(lens), Hq, H, d, page, smooth)
    run_attention(c, table, lens, starts, q, 1, True, window=window, sink=sink)


CHUNKS = [
    # lens, queries, Hq, H, d, page, smooth, what
    ([40, 3], [3, 5], 4, 2, 64, 16, False, "few queries, more queries than cache"),
    ([300], [16], 1, 1, 128, 16, True, "sixteen rows"),
    ([300], [17], 1, 1, 128, 16, True, "seventeen rows"),
    ([100, 0, 260], [33, 2, 64], 2, 2, 64, 32, True, "empty cache among others"),
    ([129, 500], [40, 129], 8, 2, 128, 48, False, "grouped heads, several blocks of rows"),
    ([700], [300], 3, 3, 128, 80, True, "more than 256 rows a head"),
    ([222, 90], [90, 90], 4, 1, 80, 16, False, "head of 80"),
    ([300], [150], 2, 1, 32, 16, True, "head of 32"),
    ([260, 31], [60, 31], 2, 2, 256, 16, True, "head of 256"),
    ([200], [140], 2, 1, 192, 32, False, "head of 192"),
    ([3000], [70], 2, 2, 64, 64, False, "split over many workgroups"),
]


@pytest.mark.parametrize("case", CHUNKS, ids=[c[-1] for c in CHUNKS])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("out_f32", [False, True])
def test_attention_of_chunks(case, causal, out_f32):
    lens, queries, Hq, H, d, page, smooth, what = case
    say("[attention] chunk", what, causal, out_f32)
    c, table, starts, q = attention_case(23, lens, queries, Hq, H, d, page, smooth, gain=2.0)
    run_attention(c, table, lens, starts, q, max(queries), causal, out_f32=out_f32)


@pytest.mark.parametrize("case", CHUNKS, ids=[c[-1] for c in CHUNKS])
@pytest.mark.parametrize("causal,window,sink", [(True, 20, 3), (True, 64, 70), (False, 100, 0), (False, 1, 17)])
def test_attention_of_chunks_in_a_window(case, causal, window, sink):
    lens, queries, Hq, H, d, page, smooth, what = case
    say("[attention] chunk window", what, causal, window, sink)
    c, table, starts, q = attention_case(24, lens, queries, Hq, H, d, page, smooth)
    run_attention(c, table, lens, starts, q, max(queries), causal, window=window, sink=sink)
