"""The activations of gated layers where they can go wrong: gates that are no numbers, gates far outside of what the exponentials
take, and gates whose activation is tiny.  Against plain evaluations in 64 bits.
"""
import math

import pytest
import torch

import paper_2605_18739_amd as nv
from tests.test_e4m3 import BF, E8M0, E4M3, F32, F64, U, act_ref, gen, randn, raw, say, values

pytestmark = pytest.mark.gpu

ACTS = [nv.ACT_SILU, nv.ACT_GELU_TANH]


@pytest.mark.parametrize("where", ["dh", "gate", "up"])
@pytest.mark.parametrize("act", ACTS)
def test_nan_in_the_backward_pass(act, where):
    """dg = dh u act'(g), du = dh act(g) and h = act(g) u are NaN where a factor is: in bf16, and with scale 255 in the blocks along
    both axes.  All other blocks are what they are without it."""
    g = gen(12)
    T, F, t, f = 300, 256, 130, 5
    dh, gu = randn(g, T, F).to(BF), randn(g, T, 2 * F).to(BF)
    clean = nv.nvfp4_gated_backward(dh.cuda(), gu.cuda(), act=act, recompute_h=True, keep_bf16=True)
    (dh if where == "dh" else gu)[t, f + (F if where == "up" else 0)] = math.nan
    bad = nv.nvfp4_gated_backward(dh.cuda(), gu.cuda(), act=act, recompute_h=True, keep_bf16=True)
    in_dg, in_du, in_h = True, where != "up", where != "dh"
    say(act, where)
    places = {f: in_dg, F + f: in_du}
    nan = torch.zeros((T, 2 * F), dtype=torch.bool)
    for column, is_nan in places.items():
        nan[t, column] = is_nan
    d, d_clean = bad[3].cpu(), clean[3].cpu()
    assert torch.equal(torch.isnan(d), nan) and torch.equal(d[~nan], d_clean[~nan])
    for q, c, blocks in ((bad[0], clean[0], [(t, column // 128) for column, n in places.items() if n]),
                         (bad[1], clean[1], [(column, t // 128) for column, n in places.items() if n]),
                         (bad[2], clean[2], [(f, t // 128)] if in_h else [])):
        want = raw(c)[1].clone()
        for at in blocks:
            want[at] = 255
        assert torch.equal(raw(q)[1], want), "scales"
        spread = (want == 255).repeat_interleave(128, 1)[:, : q.K]
        assert torch.isnan(values(q)[spread]).all() and torch.equal(raw(q)[0][~spread], raw(c)[0][~spread])


@pytest.mark.parametrize("M", [3, 80])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("half", ["gate", "up"])
def test_nan_in_the_forward_pass(act, half, M):
    """A NaN code of one row of W makes that column of the gate (or the up projection) NaN, and with it h; its block's scales are 255."""
    g = gen(M)
    F, K, f = 256, 272, 133
    A = nv.nvfp4_e4m3_quantize(randn(g, M, K).to(BF).cuda())
    W = nv.nvfp4_e4m3_quantize_2d(randn(g, 2 * F, K).to(BF).cuda(), transposed=False)[0]
    clean = nv.nvfp4_e4m3_gemm_gated(A, W, act=act, keep_h=True, keep_gate_up=True)
    codes = W.codes.view(torch.uint8).clone()
    codes[f + (F if half == "up" else 0), 7] = 0x7F
    q, h, gu = nv.nvfp4_e4m3_gemm_gated(A, nv.E4M3Tensor(codes, W.scales), act=act, keep_h=True, keep_gate_up=True)
    say(act, half, M)
    keep, keep2 = torch.arange(F) != f, torch.arange(2 * F) != f + (F if half == "up" else 0)
    assert torch.isnan(h[:, f]).all() and torch.equal(h.cpu()[:, keep], clean[1].cpu()[:, keep])
    assert torch.isnan(gu.cpu()[:, ~keep2]).all() and torch.equal(gu.cpu()[:, keep2], clean[2].cpu()[:, keep2])
    s, want = raw(q)[1], raw(clean[0])[1].clone()
    want[:, f // 128] = 255
    assert torch.equal(s, want) and torch.isnan(values(q)[:, 128:]).all() and torch.equal(raw(q)[0][:, :128], raw(clean[0])[0][:, :128])


@pytest.mark.parametrize("M", [2, 70])
@pytest.mark.parametrize("act", ACTS)
def test_gates_at_the_end_of_the_range(act, M):
    """Gates of +-1.75 * 2^127 and +-infinity times a small up value: a finite gate gives h = g u or zero, +infinity infinity; -infinity
    is NaN, as it is times the sigmoid's zero."""
    F, K = 16, 16
    v = torch.zeros((2 * F, K))
    v[:F, 0] = torch.where(torch.arange(F) % 2 == 0, 1.75, -1.75)
    v[F:, 0] = 1.0
    e = torch.tensor([67] * F + [-120] * F)                                     # gate rows times 2^67, up rows times 2^-120
    W = nv.E4M3Tensor(v.to(E4M3).cuda(), (e + 127).to(torch.uint8).view(2 * F, 1).view(E8M0).cuda())
    A = nv.E4M3Tensor(torch.nn.functional.pad(torch.ones((M, 1)), (0, K - 1)).to(E4M3).cuda(),
                      (torch.where(torch.arange(M) % 2 == 0, 60, 64) + 127).to(torch.uint8).view(M, 1).view(E8M0).cuda())
    y = values(A) @ values(W).T
    gate = y[:, :F].float().double()                                            # (2^131 is infinite in 32 bits)
    assert torch.isinf(gate[1::2]).all() and (gate[::2].abs() == 1.75 * 2.0 ** 127).all()
    q, h, _ = nv.nvfp4_e4m3_gemm_gated(A, W, act=act, keep_h=True)
    h, want = h.cpu(), act_ref(act, gate)[0] * y[:, F:]
    say(act, M)
    assert torch.equal(torch.isnan(h), torch.isnan(want))
    assert torch.equal(h[0::2].double(), want[0::2]) and torch.isposinf(h[1::2, 0::2]).all() and torch.isnan(h[1::2, 1::2]).all()      # (seven bits: exact)
    assert (raw(q)[1][1::2] == 255).all() and torch.equal(values(q)[0::2], want[0::2])


@pytest.mark.parametrize("act", ACTS)
def test_gradients_at_the_end_of_the_range(act):
    """act' is one above and zero below what the exponentials take, up to the infinities, and act is g or zero."""
    gates = torch.tensor([2.0 ** 127, 3.2e38, 2.4e38, 2.2e38, 1e30, 500.0, 105.0, 104.0, math.inf, -math.inf, -3.2e38, -2.2e38, -1e30, -500.0, -105.0, -88.0]).to(BF)
    T, F = 5, 16
    g = gen(3)
    dh, up = (1e-3 * (1 + torch.rand((T, F), generator=g))).to(BF), randn(g, T, F).to(BF)
    d = nv.nvfp4_gated_backward(dh.cuda(), torch.cat([gates.expand(T, F), up], 1).contiguous().cuda(), act=act, quantize=False, keep_bf16=True)[3].cpu().double()
    positive = gates.double() > 0
    slope, a = positive.double(), torch.where(positive, gates.double(), 0.0)
    a[9] = math.nan                                                             # -infinity times zero
    want = torch.cat([dh.double() * up.double() * slope, dh.double() * a], 1)
    # two products in 32 bits (2^-23 in all) and one rounding to bf16; below -87 the activation is taken as zero (at most 1.44e-36)
    assert torch.equal(torch.isnan(d), torch.isnan(want))
    same = torch.isinf(want) & (d == want) | torch.isnan(want)
    assert (same | ((d - want).abs() <= (2.0 ** -8 + 2.0 ** -22) * want.abs() + 1.5e-36)).all()


def assert_rounded(got, want, err, what):
    """Every bf16 number is the rounding of something within err of want: off by a rounding elsewhere does not hide what is off here."""
    low, high = (want - err).float().to(BF).double(), (want + err).float().to(BF).double()
    out = (got < low) | (got > high)
    assert not out.any(), f"{what}: {int(out.sum())} of {out.numel()} numbers round to something else, the first at {out.nonzero()[0].tolist()}"


def negative_gates(g, M, F):
    """Operands whose gates are sums of exact products, all over (-10, 0), and whose up values are one."""
    K, terms = 16, 6
    a, w = torch.zeros((M, K)), torch.zeros((2 * F, K))
    a[:, 0] = -torch.randint(8, 16, (M,), generator=g) / 8 * torch.exp2(torch.randint(-2, 3, (M,), generator=g).float())
    w[:F, 0] = torch.randint(8, 16, (F,), generator=g) / 8
    a[:, 1 : 1 + terms] = torch.randint(8, 16, (M, terms), generator=g) / 512
    w[:F, 1 : 1 + terms] = torch.randint(-15, 16, (F, terms), generator=g) / 32
    a[:, 15] = w[F:, 15] = 1.0
    one = lambda v: nv.E4M3Tensor(v.to(E4M3).cuda(), torch.full((v.shape[0], 1), 127, dtype=torch.uint8).view(E8M0).cuda())
    assert (a.to(E4M3).float() == a).all() and (w.to(E4M3).float() == w).all()
    return one(a), one(w)


@pytest.mark.parametrize("M", [50, 900])
@pytest.mark.parametrize("act", ACTS)
def test_small_activations(act, M):
    """The activation of negative gates, which is about g e^z, relative to itself.  An error of z counts |z| times there, so z may not be
    a rounded number: e^z within 2 u of the hardware's and 2 u of its exponent's parts and the product with them, a sum, a reciprocal
    and a product 4 u, and the roundings of this test's bounds to fp32: 9 u."""
    A, W = negative_gates(gen(M), M, 384)
    y = values(A) @ values(W).T
    assert (y.float().double() == y).all() and (y[:, 384:] == 1).all()
    gate = y[:, :384]
    h = nv.nvfp4_e4m3_gemm_gated(A, W, act=act, quantize=False, keep_h=True)[1].cpu().double()
    want = act_ref(act, gate)[0]
    say(act, M, "gates", float(gate.min()), float(gate.max()), "below -3:", int((gate < -3).sum()))
    inside = gate > -9.8                                                        # (further down the sigmoid of GELU leaves the normal numbers)
    assert_rounded(h[inside], want[inside], 9 * U * want[inside].abs(), "act")


@pytest.mark.parametrize("act", ACTS)
def test_gradients_of_small_activations(act):
    """As above for du = dh act(g): one product more, 10 u; and dg = dh u act'(g), act' = s + g s (1 - s) z': s and 1 - s within 6 u of
    themselves (SiLU: 1 - s within 6 u of s), z' 2 u, six products and a sum: 16 u of the sum of its terms' magnitudes."""
    g = gen(7)
    T, F = 700, 384
    gate = (-9.8 * torch.rand((T, F), generator=g)).to(BF)
    dh, up = randn(g, T, F).to(BF), randn(g, T, F).to(BF)
    d = nv.nvfp4_gated_backward(dh.cuda(), torch.cat([gate, up], 1).cuda(), act=act, quantize=False, keep_bf16=True)[3].cpu().double()
    gate, dh, up = gate.double(), dh.double(), up.double()
    a, slope = act_ref(act, gate)
    s = torch.sigmoid(gate if act == nv.ACT_SILU else math.sqrt(8 / math.pi) * (gate + 0.044715 * gate ** 3))
    inner = 1.0 if act == nv.ACT_SILU else math.sqrt(8 / math.pi) * (1 + 0.134145 * gate ** 2)
    say(act)
    assert_rounded(d[:, F:], dh * a, 10 * U * (dh * a).abs(), "du")
    assert_rounded(d[:, :F], dh * up * slope, 16 * U * (dh * up).abs() * s * (1 + gate.abs() * inner), "dg")
