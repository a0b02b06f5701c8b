"""8-bit operands: quantizers, products, gated projections and their backward pass on the GPU against plain evaluations in 64 bits.

Bounds (u = 2^-24, half an fp32 step; bf16 half step 2^-8, E4M3 2^-4 relative, 2^-10 of the block's scale below its normal numbers):
 quantizers of bf16   exact: scaling by a power of two rounds nothing, so every byte is decided by the definition.
 product              fp32 sums of K exact products in some order, each addition within a step 2^-23 of partial sums that are at
                      most S = sum |a w|: K 2^-23 S, and 2^-8 |y| for bf16.  Small integers whose sums stay below 2^24: exact.
 fast sums            of eight products seven may lose up to 2^-13 of the largest: 7 * 2^-13 < 2^-10 of their magnitudes' sum.
 gated                E_g, E_u as above; act has slope at most 1.13 and its evaluation is within 8 u (|g| + 1) of |act|, so
                      E_h = |u| (1.13 E_g + 8 u (|g| + 1) |act|) + |act| E_u + 4 u |h| + 1.13 E_g E_u; a code is the rounding of
                      something within E_h of h: E_h + 2^-4 (|h| + E_h) + 2^-10 s.
 gated backward       fp32 chains of at most 16 roundings on exact bf16 inputs: 32 u (1 + |g|) of the product of the factors'
                      magnitudes, then as above.
 scales               those of the largest magnitude, or of one within the error bound of it.
"""
import math

import pytest
import torch

import paper_2605_18739_amd as nv

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def say(*a):
    print(*a, flush=True)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape):
    return torch.randn(shape, generator=g, dtype=F32)


def ceil(n, to):
    return -(-n // to)


# ---------------------------------------------------------------------------------------------------------------------
# the definition
# ---------------------------------------------------------------------------------------------------------------------
GRID = torch.tensor([m / 512 for m in range(8)] + [(8 + m) / 8 * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1], dtype=F64)
POWERS = torch.tensor([2.0 ** e for e in range(-127, 121)], dtype=F64)


def scale_bytes(amax):
    """Blocks' largest magnitudes in 64 bits -> bytes."""
    return torch.where(torch.isfinite(amax), torch.bucketize(amax.contiguous(), 448 * POWERS), 255).to(torch.uint8)


def nearest_bytes(y):
    mid = (GRID[1:] + GRID[:-1]) / 2
    a = y.abs().contiguous()
    low, up = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)
    return (torch.where(low % 2 == 0, low, up) + 128 * torch.signbit(y)).to(torch.uint8)


def quantized(x, tile=False):
    """Matrix in 64 bits -> (code bytes, scale bytes); NaN codes compare by their magnitude bits."""
    R, K = x.shape
    rows, cols = (128 * ceil(R, 128) if tile else R), 128 * ceil(K, 128)
    p = torch.zeros((rows, cols), dtype=F64)
    p[:R, :K] = x
    a = p.abs().nan_to_num(nan=math.inf, posinf=math.inf)
    amax = a.view(rows // 128, 128, cols // 128, 128).amax((1, 3)) if tile else a.view(rows, cols // 128, 128).amax(2)
    s = scale_bytes(amax)
    e = (s.repeat_interleave(128, 0)[:R] if tile else s).repeat_interleave(128, 1)[:, :K].to(F64) - 127
    codes = nearest_bytes((x / torch.pow(torch.tensor(2.0, dtype=F64), e)).nan_to_num())
    codes[e == 128] = 0x7F
    return codes, s


def values(t):
    """What a device E4M3Tensor stands for, in 64 bits on the host."""
    codes, s = t.codes.cpu(), t.scales.cpu().to(F64)
    if t.block_rows != 1:
        s = s.repeat_interleave(128, 0)[: t.rows]
    return codes.to(F64) * s.repeat_interleave(128, 1)[:, : t.K]


def raw(t):
    return t.codes.cpu().view(torch.uint8), t.scales.cpu().view(torch.uint8)


def poisoned(rows, K, block_rows=1):
    """An output tensor inside a larger buffer of 0xEE bytes, and a check that nothing around it was written."""
    def part(n):
        whole = torch.full((n + 512,), 0xEE, dtype=torch.uint8, device="cuda")
        return whole, whole[256 : 256 + n]
    n_s = (ceil(rows, block_rows), ceil(K, 128))
    wc, c = part(rows * K)
    ws, s = part(n_s[0] * n_s[1])
    t = nv.E4M3Tensor(c.view(rows, K).view(E4M3), s.view(n_s).view(E8M0))

    def intact():
        for w, n in ((wc, rows * K), (ws, n_s[0] * n_s[1])):
            assert (w[:256] == 0xEE).all() and (w[256 + n :] == 0xEE).all(), "bytes around an output were written"
    return t, intact


def assert_exact(t, want, what):
    codes, s = raw(t)
    assert torch.equal(s, want[1]), f"{what}: scales differ at {(s != want[1]).nonzero()[0].tolist()}"
    got, ref = codes.clone(), want[0].clone()
    nan = (ref & 127) == 127
    got[nan] &= 127
    assert torch.equal(got, ref), f"{what}: codes differ at {(got != ref).nonzero()[0].tolist()}"


def strided(x, pad):
    """x on the GPU as columns of a wider matrix whose other columns are NaN."""
    if not pad:
        return x.to("cuda")
    wide = torch.full((x.shape[0], x.shape[1] + pad), math.nan, dtype=x.dtype, device="cuda")
    wide[:, 8 : 8 + x.shape[1]] = x.to("cuda")
    return wide[:, 8 : 8 + x.shape[1]]


# ---------------------------------------------------------------------------------------------------------------------
# quantizers
# ---------------------------------------------------------------------------------------------------------------------
def mixed(g, R, C):
    """Rows and columns of very different magnitudes, some of them zero."""
    x = randn(g, R, C) * torch.exp2(torch.randint(-30, 30, (R, 1), generator=g).float()) * torch.exp2(torch.randint(-8, 9, (1, C), generator=g).float())
    x[torch.rand((R, C), generator=g) < 0.05] = 0.0
    x[R // 2] = 0.0
    x[:, C // 3] = -0.0
    return x.to(BF)


@pytest.mark.parametrize("R,C,pad", [(1, 16, 0), (1, 128, 0), (3, 144, 0), (5, 512, 24), (129, 528, 0), (64, 2064, 8), (37, 14336, 0), (1000, 80, 16)])
def test_quantize_rows(R, C, pad):
    x = mixed(gen(R + C), R, C)
    out, intact = poisoned(R, C)
    assert nv.nvfp4_e4m3_quantize(strided(x, pad), out=out) is out
    assert_exact(out, quantized(x.double()), f"rows {R}x{C}")
    intact()
    assert_exact(nv.nvfp4_e4m3_quantize(strided(x, pad)), quantized(x.double()), "new output")


@pytest.mark.parametrize("R,C,pad", [(1, 8, 0), (15, 16, 0), (16, 136, 8), (127, 128, 0), (128, 256, 0), (129, 264, 24), (1000, 72, 0), (2050, 40, 0)])
def test_quantize_columns(R, C, pad):
    x = mixed(gen(R + C), R, C)
    K = 16 * ceil(R, 16)
    t = torch.zeros((C, K), dtype=F64)
    t[:, :R] = x.double().T
    out, intact = poisoned(C, K)
    nv.nvfp4_e4m3_quantize(strided(x, pad), block_axis=1, out=out)
    assert_exact(out, quantized(t), f"columns {R}x{C}")
    intact()


@pytest.mark.parametrize("R,C,pad", [(16, 16, 0), (16, 144, 8), (128, 128, 0), (144, 400, 0), (272, 112, 16), (1024, 640, 0)])
def test_quantize_tiles(R, C, pad):
    x = mixed(gen(R + C), R, C)
    (out, intact), (out_t, intact_t) = poisoned(R, C, 128), poisoned(C, R, 128)
    nv.nvfp4_e4m3_quantize_2d(strided(x, pad), out=out, out_t=out_t)
    codes, s = quantized(x.double(), tile=True)
    assert_exact(out, (codes, s), "tiles")
    assert_exact(out_t, (codes.T.contiguous(), s.T.contiguous()), "tiles, transposed")
    intact(), intact_t()
    alone, none = nv.nvfp4_e4m3_quantize_2d(strided(x, pad), transposed=False)
    assert none is None
    assert_exact(alone, (codes, s), "tiles alone")


def test_quantize_borders():
    """Largest magnitudes at, below and above 448 times a power of two, over the whole range; ties; subnormal codes; extremes."""
    bits = torch.arange(0, 0x7F80, dtype=torch.int32).to(torch.int16).view(BF)            # every finite bf16 magnitude
    x = torch.zeros((bits.numel(), 128), dtype=BF)
    g = gen(3)
    x[:] = bits[:, None] * (torch.randint(-256, 257, x.shape, generator=g) / 256.0).to(BF)
    x[:, 5] = bits
    x[:, 77] = -bits
    want = quantized(x.double())
    assert int(want[1].max()) == 247 and int(want[1].min()) == 0
    assert_exact(nv.nvfp4_e4m3_quantize(x.cuda()), want, "rows")
    rows = 16 * (x.shape[0] // 16)
    assert_exact(nv.nvfp4_e4m3_quantize(x[:rows].T.contiguous().cuda(), block_axis=1), (want[0][:rows], want[1][:rows]), "columns")


def test_quantize_ties():
    """Every midpoint between neighbouring codes, in blocks of scale one."""
    y = torch.cat([GRID, (GRID[1:] + GRID[:-1]) / 2])
    x = torch.zeros((2, 256), dtype=F64)
    x[0, : y.numel()], x[1, : y.numel()] = y, -y
    x[:, 100] = x[:, 200] = 448.0
    assert (x.to(BF).double() == x).all()
    want = quantized(x)
    assert (want[1] == 127).all()
    assert_exact(nv.nvfp4_e4m3_quantize(x.to(BF).cuda()), want, "ties")


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_quantize_not_finite(value):
    """The block that holds it becomes NaN, no other one does."""
    x = randn(gen(1), 256, 384)
    x[17, 130] = value
    x = x.to(BF)
    assert_exact(nv.nvfp4_e4m3_quantize(x.cuda()), quantized(x.double()), "rows")
    assert_exact(nv.nvfp4_e4m3_quantize(x.cuda(), block_axis=1), quantized(x.double().T.contiguous()), "columns")
    q, t = nv.nvfp4_e4m3_quantize_2d(x.cuda())
    codes, s = quantized(x.double(), tile=True)
    assert_exact(q, (codes, s), "tiles")
    assert_exact(t, (codes.T.contiguous(), s.T.contiguous()), "tiles, transposed")
    assert torch.isnan(values(q)[:128, 128:256]).all() and int(torch.isnan(values(q)).sum()) == 128 * 128


# ---------------------------------------------------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------------------------------------------------
def small_integers(g, rows, K, tile):
    """Codes -4 .. 4 and scales 1, 2, 4: products with sums below 2^24 for K <= 16384."""
    v = torch.randint(-4, 5, (rows, K), generator=g).float()
    s = torch.randint(0, 3, (ceil(rows, 128) if tile else rows, ceil(K, 128)), generator=g)
    return nv.E4M3Tensor(v.to(E4M3).cuda(), (s + 127).to(torch.uint8).view(E8M0).cuda())


def real_operand(g, rows, K, tile):
    x = (randn(g, rows, K) * torch.exp2(torch.randint(-3, 4, (1, K), generator=g).float())).to(BF)
    codes, s = quantized(x.double(), tile)
    return nv.E4M3Tensor(codes.view(E4M3).cuda(), s.view(E8M0).cuda())


SHAPES = [(1, 1, 16), (1, 16, 128), (2, 7, 144), (3, 50, 1040), (16, 33, 2000), (17, 128, 4096), (33, 200, 512), (64, 1111, 400), (65, 129, 272), (100, 100, 16),
          (129, 1, 640), (128, 256, 1024), (200, 300, 656), (257, 513, 1040), (777, 1111, 2000), (1025, 2050, 384), (4097, 1030, 528), (3500, 4000, 272), (2, 14336, 128)]


@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_integers(M, N, K, tile):
    g = gen(M + N + K)
    A, W = small_integers(g, M, K, False), small_integers(g, N, K, tile)
    want = (values(A).float() @ values(W).float().T).double()       # (exact: integers below 2^24)
    y = nv.nvfp4_e4m3_gemm(A, W)
    say(M, N, K, tile)
    assert torch.equal(y.cpu().double(), want)
    assert torch.equal(nv.nvfp4_e4m3_gemm(A, W, fast_sums=True).cpu().double(), want)      # (no product of eight is 2^13 times another)
    assert torch.equal(nv.nvfp4_e4m3_gemm(A, W, out_dtype=nv.OUT_BF16).cpu(), want.float().to(BF))


@pytest.mark.parametrize("M,N,K,tile", [(5, 300, 14336, True), (40, 130, 2000, False), (300, 200, 17600, False), (777, 1111, 2000, True), (2100, 4100, 640, True)])
def test_gemm_rounding(M, N, K, tile):
    g = gen(M + N + K)
    A, W = real_operand(g, M, K, False), real_operand(g, N, K, tile)
    a, w = values(A), values(W)
    want, S = a @ w.T, a.abs() @ w.abs().T
    y = nv.nvfp4_e4m3_gemm(A, W).cpu().double()
    say("relative error", float((y - want).norm() / want.norm()), "worst of sum |a w|", float(((y - want).abs() / S).max()))
    assert ((y - want).abs() <= K * 2 * U * S).all()
    b = nv.nvfp4_e4m3_gemm(A, W, out_dtype=nv.OUT_BF16).cpu().double()
    assert ((b - want).abs() <= K * 2 * U * S * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()).all()
    f = nv.nvfp4_e4m3_gemm(A, W, fast_sums=True).cpu().double()
    say("fast sums: relative error", float((f - want).norm() / want.norm()), "worst of sum |a w|", float(((f - want).abs() / S).max()))
    assert ((f - want).abs() <= (K * 2 * U + 2.0 ** -10) * S).all()


@pytest.mark.parametrize("dtype", [nv.OUT_F32, nv.OUT_BF16])
@pytest.mark.parametrize("M,N,ld,first", [(70, 100, 133, 3), (70, 100, 136, 8), (300, 257, 300, 1), (9, 40, 57, 5), (600, 1000, 1024, 16)])
def test_gemm_into_columns(M, N, ld, first, dtype):
    """Outputs inside wider matrices at any place: what is around them stays."""
    g = gen(M + N)
    A, W = small_integers(g, M, 272, False), small_integers(g, N, 272, True)
    whole = torch.full((M, ld), 7.0, dtype=F32 if dtype == nv.OUT_F32 else BF, device="cuda")
    Y = whole[:, first : first + N]
    assert nv.nvfp4_e4m3_gemm(A, W, out_dtype=dtype, Y=Y) is Y
    want = (values(A).float() @ values(W).float().T).to(whole.dtype)
    assert torch.equal(Y.cpu(), want)
    assert (whole[:, :first] == 7).all() and (whole[:, first + N :] == 7).all()


@pytest.mark.parametrize("M,fast", [(3, False), (200, False), (200, True)])
def test_gemm_scales(M, fast):
    """Scales over the whole range; a NaN scale and a NaN code reach their own row or columns and no others."""
    g = gen(5)
    A, W = small_integers(g, M, 512, False), small_integers(g, 256, 512, True)
    e = torch.randint(-40, 40, (M, 1), generator=g)
    A = nv.E4M3Tensor(A.codes, (e + 127).expand(M, 4).contiguous().to(torch.uint8).view(E8M0).cuda())
    W = nv.E4M3Tensor(W.codes, torch.tensor([[67] * 4, [187] * 4], dtype=torch.uint8).view(E8M0).cuda())
    want = A.codes.cpu().float() @ W.codes.cpu().float().T                      # integers, then one power of two for each result
    want = want.double() * torch.exp2(e.double()) * torch.exp2(torch.tensor([-60.0] * 128 + [60.0] * 128, dtype=F64))
    assert torch.equal(nv.nvfp4_e4m3_gemm(A, W, fast_sums=fast).cpu().double(), want)
    s = A.scales.view(torch.uint8).clone()
    s[1, 3] = 255
    bad = nv.nvfp4_e4m3_gemm(nv.E4M3Tensor(A.codes, s), W, fast_sums=fast).cpu().double()
    assert torch.isnan(bad[1]).all()
    keep = torch.arange(M) != 1
    assert torch.equal(bad[keep], want[keep])
    c = W.codes.view(torch.uint8).clone()
    c[130, 511] = 0x7F
    bad = nv.nvfp4_e4m3_gemm(A, nv.E4M3Tensor(c, W.scales), fast_sums=fast).cpu().double()
    keep = torch.arange(256) != 130
    assert torch.isnan(bad[:, 130]).all() and torch.equal(bad[:, keep], want[:, keep])


# ---------------------------------------------------------------------------------------------------------------------
# gated projections
# ---------------------------------------------------------------------------------------------------------------------
def act_ref(act, g):
    """act(g) and its derivative in 64 bits."""
    if act == nv.ACT_SILU:
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * torch.sigmoid(-g))
    z = math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3)
    s = torch.sigmoid(z)
    return g * s, s * (1 + g * torch.sigmoid(-z) * math.sqrt(8 / math.pi) * (1 + 0.134145 * g ** 2))


def assert_codes(t, want, err, what):
    """t holds roundings of numbers within err of want, with a scale that such numbers have."""
    rows, K = want.shape
    cols = 128 * ceil(K, 128)
    p, q = torch.zeros((2, rows, cols), dtype=F64)
    p[:, :K], q[:, :K] = (want.abs() - err).clamp(min=0), want.abs() + err
    low, high = (scale_bytes(v.view(rows, -1, 128).amax(2)) for v in (p, q))
    s = raw(t)[1]
    assert ((s >= low) & (s <= high)).all(), f"{what}: a scale is off"
    unit = torch.exp2(s.double() - 127).repeat_interleave(128, 1)[:, :K]
    off = (values(t) - want).abs()
    bound = err + 2.0 ** -4 * (want.abs() + err) + 2.0 ** -10 * unit
    assert (off <= bound).all(), f"{what}: {float((off / bound).max())} of the bound"


@pytest.mark.parametrize("act", [nv.ACT_SILU, nv.ACT_GELU_TANH])
@pytest.mark.parametrize("M,F,K,tile", [(1, 16, 16, True), (5, 400, 1040, True), (20, 144, 2000, False), (64, 256, 512, True), (65, 128, 272, True), (130, 272, 640, False),
                                        (300, 1008, 528, True), (1030, 1040, 400, True), (1100, 4112, 272, True)])
def test_gated(M, F, K, tile, act):
    g = gen(M + F + K)
    A = real_operand(g, M, K, False)
    W0 = real_operand(g, 2 * F, K, tile)
    W = nv.E4M3Tensor(W0.codes, (W0.scales.view(torch.uint8).int() - 2 - int(math.log2(K) / 2)).to(torch.uint8).view(E8M0))
    a, w = values(A), values(W)
    y, S = a @ w.T, a.abs() @ w.abs().T
    E = K * 2 * U * S
    gate, up, Eg, Eu = y[:, :F], y[:, F:], E[:, :F], E[:, F:]
    s = act_ref(act, gate)[0]
    h = s * up
    Eh = up.abs() * (1.13 * Eg + 8 * U * (gate.abs() + 1) * s.abs()) + s.abs() * Eu + 4 * U * h.abs() + 1.13 * Eg * Eu
    out, intact = poisoned(M, F)
    wide = torch.full((M, 2 * F + 11), 7.0, dtype=BF, device="cuda")
    gate_up = wide[:, 3 : 3 + 2 * F]
    o, h_bf16, gu = nv.nvfp4_e4m3_gemm_gated(A, W, act=act, out=out, keep_h=True, gate_up=gate_up)
    assert o is out and gu is gate_up
    say(M, F, K, tile, act)
    assert_codes(out, h, Eh, "h")
    intact()
    assert ((h_bf16.cpu().double() - h).abs() <= Eh + 2.0 ** -8 * (h.abs() + Eh)).all()
    assert ((gu.cpu().double() - y).abs() <= E + 2.0 ** -8 * (y.abs() + E)).all()
    assert (wide[:, :3] == 7).all() and (wide[:, 3 + 2 * F :] == 7).all()
    alone, none, none_too = nv.nvfp4_e4m3_gemm_gated(A, W, act=act)
    assert none is None and none_too is None
    assert all(torch.equal(x, z) for x, z in zip(raw(alone), raw(out)))
    no_codes, h_alone, _ = nv.nvfp4_e4m3_gemm_gated(A, W, act=act, quantize=False, keep_h=True)
    assert no_codes is None and torch.equal(h_alone, h_bf16)


@pytest.mark.parametrize("M,F", [(3, 37), (70, 37), (130, 1), (20, 129), (300, 263)])
def test_gated_of_odd_widths(M, F):
    """Without an 8-bit result F may be anything: the gate's and the up projection's rows meet inside a block of scales."""
    g = gen(M + F)
    A, W = small_integers(g, M, 400, False), small_integers(g, 2 * F, 400, True)
    y = values(A) @ values(W).T
    none, h, gu = nv.nvfp4_e4m3_gemm_gated(A, W, quantize=False, keep_h=True, keep_gate_up=True)
    assert none is None and torch.equal(gu.cpu(), y.float().to(BF))
    want = act_ref(nv.ACT_SILU, y[:, :F])[0] * y[:, F:]                         # (exact sums; the activation within 8 u (|g| + 1))
    # (gates here are integers up to thousands.  Below -87 the sigmoid, then under e^-87 = 1.65e-38, the least normal number's
    #  neighbourhood, is taken as zero: |g| e^-|g| falls from there on, so h is off by at most 87 * 1.65e-38 |u| = 1.44e-36 |u|)
    E = 8 * U * (y[:, :F].abs() + 1) * want.abs() + 4 * U * want.abs() + 1.44e-36 * y[:, F:].abs() + 1e-36
    assert ((h.cpu().double() - want).abs() <= E + 2.0 ** -8 * (want.abs() + E)).all()


def test_gated_fast_sums():
    """The 8-bit instruction's sums in the gated form: exact for small integers, and so the same bytes."""
    g = gen(21)
    A, W = small_integers(g, 200, 512, False), small_integers(g, 2 * 272, 512, True)
    W = nv.E4M3Tensor(W.codes, (W.scales.view(torch.uint8) - 9).view(E8M0))
    exact, fast = (nv.nvfp4_e4m3_gemm_gated(A, W, keep_h=True, keep_gate_up=True, fast_sums=f) for f in (False, True))
    assert all(torch.equal(x, y) for x, y in zip(raw(exact[0]), raw(fast[0]))) and torch.equal(exact[1], fast[1]) and torch.equal(exact[2], fast[2])


@pytest.mark.parametrize("M,N,K", [(4097, 1030, 2032), (4097, 1030, 1680), (4352, 1900, 1808), (4352, 1900, 1152), (300, 700, 1984), (300, 700, 1424)])
def test_products_over_several_turns(M, N, K):
    """Stages of LDS change places from turn to turn (four steps of 128 k): whole turns and parts of one, tiles of each kind."""
    g = gen(M + K)
    A, W = small_integers(g, M, K, False), small_integers(g, N, K, True)
    want = values(A).float() @ values(W).float().T                  # (exact: integers below 2^24)
    say(M, N, K)
    for fast in (False, True):
        assert torch.equal(nv.nvfp4_e4m3_gemm(A, W, fast_sums=fast).cpu(), want), fast


@pytest.mark.parametrize("K", [512, 1424, 2032])
def test_gated_fast_sums_over_several_turns(K):
    """As test_gated_fast_sums, at sizes that take tiles of 128 x 256."""
    g = gen(K)
    A, W = small_integers(g, 1100, K, False), small_integers(g, 2 * 2700, K, True)
    W = nv.E4M3Tensor(W.codes, (W.scales.view(torch.uint8) - 9).view(E8M0))
    say(K)
    exact, fast = (nv.nvfp4_e4m3_gemm_gated(A, W, quantize=False, keep_h=True, keep_gate_up=True, fast_sums=f) for f in (False, True))
    assert torch.equal(exact[1], fast[1]) and torch.equal(exact[2], fast[2])


def test_gated_of_large_gates():
    """Gates far outside of what the exponentials take: h goes to zero or to g u, and stays finite."""
    K, F = 16, 16
    A = nv.E4M3Tensor(torch.full((3, K), 1.0).to(E4M3).cuda(), torch.tensor([[127], [137], [187]], dtype=torch.uint8).view(E8M0).cuda())
    v = torch.zeros((2 * F, K))
    v[:F] = torch.where(torch.arange(F) % 2 == 0, 1.0, -1.0)[:, None]
    v[F:] = 0.5
    W = nv.E4M3Tensor(v.to(E4M3).cuda(), torch.full((2 * F, 1), 127, dtype=torch.uint8).view(E8M0).cuda())
    y = values(A) @ values(W).T
    for act in (nv.ACT_SILU, nv.ACT_GELU_TANH):
        h = nv.nvfp4_e4m3_gemm_gated(A, W, act=act, keep_h=True)[1].cpu().double()
        want = act_ref(act, y[:, :F])[0] * y[:, F:]
        assert torch.isfinite(h).all()
        assert ((h - want).abs() <= (2.0 ** -8 + 2.0 ** -12) * want.abs() + 1e-36).all()


# ---------------------------------------------------------------------------------------------------------------------
# the gated activation's backward pass
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("act", [nv.ACT_SILU, nv.ACT_GELU_TANH])
@pytest.mark.parametrize("T,F,pad", [(1, 128, 0), (15, 256, 0), (16, 128, 24), (130, 384, 0), (129, 128, 8), (700, 640, 0)])
def test_gated_backward(T, F, pad, act):
    g = gen(T + F)
    dh, gu = (1e-3 * randn(g, T, F)).to(BF), (1.5 * randn(g, T, 2 * F)).to(BF)
    gu[0, :4], gu[-1, F : F + 4] = torch.tensor([30.0, -30.0, 200.0, -200.0]).to(BF), 0.0
    gate, up, d = gu[:, :F].double(), gu[:, F:].double(), dh.double()
    a, slope = act_ref(act, gate)
    want = torch.cat([d * up * slope, d * a], 1)
    h = a * up
    E = 32 * U * torch.cat([(d * up).abs() * (1 + gate.abs()), d.abs() * (a.abs() * (1 + gate.abs()))], 1) + 1e-38
    Eh = 32 * U * (a * up).abs() * (1 + gate.abs()) + 1e-38
    T16 = 16 * ceil(T, 16)
    (o, i0), (o_t, i1), (h_t, i2) = poisoned(T, 2 * F), poisoned(2 * F, T16), poisoned(F, T16)
    got = nv.nvfp4_gated_backward(strided(dh, pad), strided(gu, pad), act=act, out=o, out_t=o_t, h_t=h_t, keep_bf16=True)
    assert got[0] is o and got[1] is o_t and got[2] is h_t
    say(T, F, act)

    def turned(x):
        t = torch.zeros((x.shape[1], T16), dtype=F64)
        t[:, :T] = x.T
        return t
    assert_codes(o, want, E, "along the features")
    assert_codes(o_t, turned(want), turned(E), "along the tokens")
    assert_codes(h_t, turned(h), turned(Eh), "h along the tokens")
    assert (raw(o_t)[0][:, T:] & 127 == 0).all() and (raw(h_t)[0][:, T:] & 127 == 0).all()
    assert ((got[3].cpu().double() - want).abs() <= E + 2.0 ** -8 * (want.abs() + E)).all()
    i0(), i1(), i2()
    in_place = gu.cuda()
    assert nv.nvfp4_gated_backward(dh.cuda(), in_place, act=act, quantize=False, d=in_place)[3] is in_place
    assert torch.equal(in_place, got[3])


@pytest.mark.parametrize("T,F", [(40, 8), (130, 136), (257, 264)])
def test_gated_backward_of_odd_widths(T, F):
    """Along the tokens F may be any multiple of eight; one result alone is what it is beside the others."""
    g = gen(T + F)
    dh, gu = randn(g, T, F).to(BF), (1.5 * randn(g, T, 2 * F)).to(BF)
    gate, up, d = gu[:, :F].double(), gu[:, F:].double(), dh.double()
    a, slope = act_ref(nv.ACT_SILU, gate)
    T16 = 16 * ceil(T, 16)

    def turned(x):
        t = torch.zeros((x.shape[1], T16), dtype=F64)
        t[:, :T] = x.T
        return t
    want, E = torch.cat([d * up * slope, d * a], 1), 32 * U * torch.cat([(d * up).abs(), (d * a).abs()], 1) * (1 + gate.abs()).repeat(1, 2) + 1e-38
    (o_t, i1), (h_t, i2) = poisoned(2 * F, T16), poisoned(F, T16)
    nv.nvfp4_gated_backward(dh.cuda(), gu.cuda(), quantize=False, out_t=o_t, h_t=h_t)
    assert_codes(o_t, turned(want), turned(E), "along the tokens")
    assert_codes(h_t, turned(a * up), turned(32 * U * (a * up).abs() * (1 + gate.abs()) + 1e-38), "h")
    i1(), i2()
    for kind in ("out_t", "h_t"):
        t, intact = poisoned(2 * F if kind == "out_t" else F, T16)
        nv.nvfp4_gated_backward(dh.cuda(), gu.cuda(), quantize=False, **{kind: t})
        assert all(torch.equal(x, y) for x, y in zip(raw(t), raw(o_t if kind == "out_t" else h_t)))
        intact()


def test_gated_backward_against_differences():
    """The gradients are those of the forward formula: central differences in 64 bits around the bf16 inputs."""
    g = gen(9)
    T, F, step = 32, 136, 1e-5
    dh, gu = randn(g, T, F).to(BF), (2 * randn(g, T, 2 * F)).to(BF)
    for act in (nv.ACT_SILU, nv.ACT_GELU_TANH):
        d = nv.nvfp4_gated_backward(dh.cuda(), gu.cuda(), act=act, quantize=False, keep_bf16=True)[3].cpu().double()

        def h(gate, up):
            return act_ref(act, gate)[0] * up
        gate, up = gu[:, :F].double(), gu[:, F:].double()
        by_gate = dh.double() * (h(gate + step, up) - h(gate - step, up)) / (2 * step)
        by_up = dh.double() * (h(gate, up + step) - h(gate, up - step)) / (2 * step)
        want = torch.cat([by_gate, by_up], 1)
        # a central difference is off by step^2 / 6 of the third derivative (below 4 of the other factor and 1) and by the rounding
        # of the differences, 2^-50 (|x| + 1)^2 / step; the kernel by its bound: 32 u (1 + |g|) of the factors, and bf16
        other = dh.double().abs().repeat(1, 2) * (1 + gate.abs().repeat(1, 2)) * (1 + up.abs().repeat(1, 2))
        assert ((d - want).abs() <= 2.0 ** -8 * want.abs() + other * (32 * U + step ** 2 + 2.0 ** -50 / step * (1 + gate.abs().repeat(1, 2)))).all()
