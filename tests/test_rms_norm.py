"""RMS norm of the residual stream and its gradient on the GPU against plain evaluations in 64 bits.

Bounds (u = 2^-24; bf16 half step 2^-8, E4M3 2^-4 relative, 2^-10 of the block's scale below its normal numbers):
 sum       exact: RN_bf16 of the two bf16 numbers' sum, which fp32 holds within half a step of its own; a tie of the second rounding
           is the first one's only where the sum is exact, so the test takes the two roundings as they are defined, fp32 first.
 y         mean of squares: at most ceil(C / L) + 10 rounded additions a lane tree of L >= 64 lanes, all of one sign, (C / 64 + 12) u
           relative, halved by the root; root 2 u, two products 2 u:  E = ((C / 64 + 12) / 2 + 5) u |y|.
 dx        r (w dy - xh m): with G = |w dy| and M = mean |w dy xh|:  r (G + |xh| M) (2 (C / 64 + 12) + 16) u, and bf16.
 dweight   (T + C / 64 + 80) u sum |dy xh|.
"""
import math

import pytest
import torch

import paper_2605_18739_amd as nv
from tests.test_e4m3 import BF, F32, F64, U, assert_codes, gen, poisoned, randn, say, strided

pytestmark = pytest.mark.gpu

EPS = 1e-6
SHAPES = [(1, 16, 0), (1, 128, 8), (5, 144, 0), (4, 512, 0), (7, 528, 24), (130, 1024, 0), (3, 1040, 0), (9, 2048, 8), (33, 2064, 0), (2, 4096, 0), (5, 5120, 16), (3, 6160, 0),
          (2, 8192, 0), (3, 8208, 0), (2, 16384, 8), (1030, 64, 0)]


def stream(g, T, C):
    """Rows of very different magnitudes with some outlier channels, and one row of zeros."""
    x = randn(g, T, C) * torch.exp2(torch.randint(-20, 20, (T, 1), generator=g).float())
    x *= torch.where(torch.rand(C, generator=g) < 0.03, 30.0, 1.0)
    if T > 2:
        x[T // 2] = 0.0
    return x.to(BF)


def norm_ref(s, w, eps=EPS):
    s, w = s.double(), w.double()
    return s / torch.sqrt(s.square().mean(1, keepdim=True) + eps) * w


def slack(C):
    return ((C / 64 + 12) / 2 + 5) * U


@pytest.mark.parametrize("T,C,pad", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_forward(T, C, pad, residual):
    g = gen(T + C)
    x, r, w = stream(g, T, C), stream(g, T, C), (1 + 0.3 * randn(g, C)).to(BF)
    s = (x.float() + r.float()).to(BF) if residual else x
    want = norm_ref(s, w)
    E = slack(C) * want.abs()
    out, intact = poisoned(T, C)
    got = nv.nvfp4_rms_norm(strided(x, pad), w.cuda(), strided(r, 2 * pad) if residual else None, eps=EPS, out=out, keep_bf16=True)
    say(T, C, pad, residual)
    assert got[0] is out
    assert_codes(out, want, E, "codes")
    intact()
    assert ((got[1].cpu().double() - want).abs() <= E + 2.0 ** -8 * (want.abs() + E)).all()
    assert torch.equal(got[2].cpu(), s) if residual else got[2] is None
    # one output alone: the same bytes
    q, none, _ = nv.nvfp4_rms_norm(strided(x, pad), w.cuda(), r.cuda() if residual else None, eps=EPS)
    assert none is None and torch.equal(q.codes.view(torch.uint8), out.codes.view(torch.uint8)) and torch.equal(q.scales.view(torch.uint8), out.scales.view(torch.uint8))
    none, y, _ = nv.nvfp4_rms_norm(strided(x, pad), w.cuda(), r.cuda() if residual else None, eps=EPS, quantize=False, keep_bf16=True)
    assert none is None and torch.equal(y, got[1])


@pytest.mark.parametrize("into", ["x", "residual"])
def test_sum_in_place(into):
    """The stream is updated where it stands, inside a wider buffer."""
    g = gen(4)
    x, r, w = stream(g, 37, 1040), stream(g, 37, 1040), (1 + 0.3 * randn(g, 1040)).to(BF)
    dx, dr = strided(x, 32), strided(r, 32)
    q, y, s = nv.nvfp4_rms_norm(dx, w.cuda(), dr, keep_bf16=True, sum=dx if into == "x" else dr)
    assert s is (dx if into == "x" else dr)
    want = (x.float() + r.float()).to(BF)
    assert torch.equal(s.cpu(), want)
    assert torch.equal((dr if into == "x" else dx).cpu(), r if into == "x" else x)
    again = nv.nvfp4_rms_norm(want.cuda(), w.cuda(), keep_bf16=True)
    assert torch.equal(again[1], y) and torch.equal(again[0].codes.view(torch.uint8), q.codes.view(torch.uint8))


def backward_ref(dy, s, w, dsum, eps=EPS):
    C = s.shape[1]
    s, g = s.double(), dy.double() * w.double()
    r = 1 / torch.sqrt(s.square().mean(1, keepdim=True) + eps)
    xh = s * r
    dx = r * (g - xh * (g * xh).mean(1, keepdim=True))
    E = r * (g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True)) * (2 * (C / 64 + 12) + 16) * U
    if dsum is not None:
        dx = dx + dsum.double()
        E = E + 2 * U * dx.abs()
    terms = dy.double() * xh
    return dx, E, terms.sum(0), (s.shape[0] + C / 64 + 80) * U * terms.abs().sum(0)


@pytest.mark.parametrize("T,C,pad", SHAPES + [(1500, 1024, 0), (2100, 2048, 0)])
@pytest.mark.parametrize("dsum", [False, True])
def test_backward(T, C, pad, dsum):
    g = gen(T + C)
    s, w = stream(g, T, C), (1 + 0.3 * randn(g, C)).to(BF)
    dy, ds = (1e-3 * randn(g, T, C)).to(BF), (1e-2 * randn(g, T, C)).to(BF) if dsum else None
    want, E, dw, Ew = backward_ref(dy, s, w, ds)
    dx, dweight = nv.nvfp4_rms_norm_backward(strided(dy, pad), strided(s, 2 * pad), w.cuda(), ds if ds is None else strided(ds, pad), eps=EPS)
    say(T, C, pad, dsum)
    assert ((dx.cpu().double() - want).abs() <= E + 2.0 ** -8 * (want.abs() + E) + 1e-38).all()
    assert ((dweight.cpu().double() - dw).abs() <= Ew + U * dw.abs() + 1e-38).all()
    alone, none = nv.nvfp4_rms_norm_backward(strided(dy, pad), s.cuda(), w.cuda(), ds if ds is None else ds.cuda(), eps=EPS, weight_grad=False)
    assert none is None and torch.equal(alone, dx)
    assert torch.equal(nv.nvfp4_rms_norm_backward(dy.cuda(), s.cuda(), w.cuda(), None if ds is None else ds.cuda(), eps=EPS)[1], dweight)


@pytest.mark.parametrize("over", ["dy", "s", "dsum"])
def test_backward_in_place(over):
    g = gen(6)
    T, C = 70, 2064
    t = {"dy": (1e-3 * randn(g, T, C)).to(BF).cuda(), "s": stream(g, T, C).cuda(), "dsum": (1e-2 * randn(g, T, C)).to(BF).cuda()}
    w = (1 + 0.3 * randn(g, C)).to(BF).cuda()
    dx, dw = nv.nvfp4_rms_norm_backward(t["dy"], t["s"], w, t["dsum"])
    same, dw2 = nv.nvfp4_rms_norm_backward(t["dy"], t["s"], w, t["dsum"], dx=t[over])
    assert same is t[over] and torch.equal(same, dx) and torch.equal(dw, dw2)


def test_backward_against_differences():
    """The gradients are those of the forward formula: central differences of sum(y dy) + sum(s dsum) in 64 bits."""
    g = gen(8)
    T, C, step = 3, 32, 1e-6
    s, w = randn(g, T, C).to(BF), (1 + 0.3 * randn(g, C)).to(BF)
    dy, ds = randn(g, T, C).to(BF), randn(g, T, C).to(BF)
    dx, dw = nv.nvfp4_rms_norm_backward(dy.cuda(), s.cuda(), w.cuda(), ds.cuda(), eps=0.1)

    def f(s, w):
        return (norm_ref(s, w, 0.1) * dy.double()).sum() + (s * ds.double()).sum()
    by_s, by_w = torch.empty((T, C), dtype=F64), torch.empty(C, dtype=F64)
    for i in range(T * C):
        e = torch.zeros(T * C, dtype=F64)
        e[i] = step
        e = e.view(T, C)
        by_s.view(-1)[i] = (f(s.double() + e, w.double()) - f(s.double() - e, w.double())) / (2 * step)
    for i in range(C):
        e = torch.zeros(C, dtype=F64)
        e[i] = step
        by_w[i] = (f(s.double(), w.double() + e) - f(s.double(), w.double() - e)) / (2 * step)
    # differences: step^2 times a third derivative below 2^8, and 2^-52 of a sum below 2^9, over the step
    slack_ = 2.0 ** 8 * step ** 2 + 2.0 ** -43 / step
    _, E, _, Ew = backward_ref(dy, s, w, ds, 0.1)
    assert ((dx.cpu().double() - by_s).abs() <= E + 2.0 ** -8 * (by_s.abs() + E) + slack_).all()
    assert ((dw.cpu().double() - by_w).abs() <= Ew + U * by_w.abs() + slack_).all()


def test_not_finite_rows_stay_alone():
    """A row with an infinity or NaN becomes NaN, the others are what they are without it."""
    g = gen(2)
    x, w = stream(g, 8, 1040), (1 + 0.3 * randn(g, 1040)).to(BF)
    clean = nv.nvfp4_rms_norm(x.cuda(), w.cuda(), keep_bf16=True)
    x[2, 7], x[5, 1000] = math.inf, math.nan
    q, y, _ = nv.nvfp4_rms_norm(x.cuda(), w.cuda(), keep_bf16=True)
    keep = [0, 1, 3, 4, 6, 7]
    assert torch.equal(y[keep], clean[1][keep]) and torch.equal(q.codes.view(torch.uint8)[keep], clean[0].codes.view(torch.uint8)[keep])
    assert torch.isnan(y[5]).all() and torch.isnan(y[2, 7])
    codes = q.codes.view(torch.uint8).cpu()
    assert (codes[5] & 127 == 127).all() and codes[2, 7] & 127 == 127
