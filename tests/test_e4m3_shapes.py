"""Every kernel that the rule of the 8-bit products can choose, over several turns of its loop, and kernels whose workgroups go from
tile to tile or from row to row, over several of those.  Bounds: tests/test_e4m3.py and tests/test_rms_norm.py.

tests/test_e4m3_plan.py checks on the CPU that the sizes below reach every kernel.
"""
import pytest
import torch

import paper_2605_18739_amd as nv
from tests.test_e4m3 import BF, E8M0, F32, F64, U, act_ref, assert_codes, ceil, gen, poisoned, randn, raw, say, small_integers, values
from tests.test_rms_norm import EPS, backward_ref, stream

pytestmark = pytest.mark.gpu

K = 1168                                               # nine steps of 128 and a part of one: two turns of four steps, and two steps more
# (M, N): every tile shape with as many stages of LDS as it can have, exact and fast sums; ends inside a tile both ways
PLAIN = [(70, 50), (80, 16460), (150, 16460), (300, 16500), (390, 18760), (400, 16460), (520, 19700), (600, 19700), (8230, 810)]
# (M, F)
GATED = [(70, 48), (80, 16464), (150, 16464), (210, 16464), (8230, 672)]
# (M, N or F) of up to 64 rows: 16, 32 and 64 rows, workgroups for one round of compute units and for more
FEW = [(M, N) for M in (8, 20, 50) for N in (400, 4112)]


def lowered(W):
    """The same codes with scales 2^9 lower: gates of a few units."""
    return nv.E4M3Tensor(W.codes, (W.scales.view(torch.uint8) - 9).view(E8M0))


@pytest.mark.parametrize("M,N", PLAIN + FEW)
def test_products_of_every_kernel(M, N):
    g = gen(M + N)
    A, W = small_integers(g, M, K, False), small_integers(g, N, K, True)
    want = values(A).float() @ values(W).float().T                  # (exact: integers below 2^24)
    say(M, N)
    for fast in (False, True):
        assert torch.equal(nv.nvfp4_e4m3_gemm(A, W, fast_sums=fast).cpu(), want), fast
        assert torch.equal(nv.nvfp4_e4m3_gemm(A, W, out_dtype=nv.OUT_BF16, fast_sums=fast).cpu(), want.to(BF)), fast


@pytest.mark.parametrize("act", [nv.ACT_SILU, nv.ACT_GELU_TANH])
@pytest.mark.parametrize("M,F", GATED + FEW)
def test_gated_products_of_every_kernel(M, F, act):
    """Sums are exact here, so gate and up values are, and h is off by the activation (8 u (|g| + 1)) and the products."""
    g = gen(M + F)
    A, W = small_integers(g, M, K, False), lowered(small_integers(g, 2 * F, K, True))
    y = (values(A).float() @ values(W).float().T).double()
    gate, up = y[:, :F], y[:, F:]
    a = act_ref(act, gate)[0]
    want = a * up
    E = up.abs() * (8 * U * (gate.abs() + 1) * a.abs() + 1.44e-36) + 4 * U * want.abs()
    say(M, F, act)
    for fast in (False, True):
        out, intact = poisoned(M, F)
        wide = torch.full((M, 2 * F + 8), 7.0, dtype=BF, device="cuda")
        _, h, gu = nv.nvfp4_e4m3_gemm_gated(A, W, act=act, out=out, keep_h=True, gate_up=wide[:, : 2 * F], fast_sums=fast)
        assert torch.equal(gu.cpu(), y.float().to(BF)) and (wide[:, 2 * F :] == 7).all()
        assert ((h.cpu().double() - want).abs() <= E + 2.0 ** -8 * (want.abs() + E)).all()
        assert_codes(out, want, E, f"fast {fast}")
        intact()


# ---------------------------------------------------------------------------------------------------------------------
# workgroups of several tiles or rows
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("act", [nv.ACT_SILU, nv.ACT_GELU_TANH])
@pytest.mark.parametrize("T,F", [(2100, 4104), (2100, 4224), (40000, 136)])
def test_gated_backward_from_tile_to_tile(T, F, act):
    """More tiles of 128 x 128 than 512: every workgroup takes a second one, some a third; with d over gate_up, too."""
    assert ceil(T, 128) * ceil(F, 128) > 512
    g = gen(T + F)
    dh, gu = (1e-3 * randn(g, T, F)).to(BF), (1.5 * randn(g, T, 2 * F)).to(BF)
    gate, up, d = gu[:, :F].double(), gu[:, F:].double(), dh.double()
    a, slope = act_ref(act, gate)
    want, h = torch.cat([d * up * slope, d * a], 1), a * up
    E = 32 * U * torch.cat([(d * up).abs() * (1 + gate.abs()), d.abs() * (a.abs() * (1 + gate.abs()))], 1) + 1e-38
    Eh = 32 * U * h.abs() * (1 + gate.abs()) + 1e-38
    T16 = 16 * ceil(T, 16)

    def turned(x):
        t = torch.zeros((x.shape[1], T16), dtype=F64)
        t[:, :T] = x.T
        return t
    say(T, F, act)
    along = F % 128 == 0
    o, o_t, h_t = poisoned(T, 2 * F) if along else (None, None), poisoned(2 * F, T16), poisoned(F, T16)
    got = nv.nvfp4_gated_backward(dh.cuda(), gu.cuda(), act=act, quantize=False, out=o[0], out_t=o_t[0], h_t=h_t[0], keep_bf16=True)[3]
    assert ((got.cpu().double() - want).abs() <= E + 2.0 ** -8 * (want.abs() + E)).all()
    if along:
        assert_codes(o[0], want, E, "along the features")
        o[1]()
    assert_codes(o_t[0], turned(want), turned(E), "along the tokens")
    assert_codes(h_t[0], turned(h), turned(Eh), "h along the tokens")
    o_t[1](), h_t[1]()
    in_place, t2 = gu.cuda(), poisoned(2 * F, T16)
    assert nv.nvfp4_gated_backward(dh.cuda(), in_place, act=act, quantize=False, out_t=t2[0], d=in_place)[3] is in_place
    assert torch.equal(in_place, got) and all(torch.equal(x, y) for x, y in zip(raw(t2[0]), raw(o_t[0])))
    t2[1]()


@pytest.mark.parametrize("T,C", [(9000, 64), (9001, 512), (8500, 1024), (1100, 5120), (600, 8208), (600, 16384)])
def test_norm_gradients_from_row_to_row(T, C):
    """Every workgroup (rows of up to 1024 elements: every wave) takes a second row, and its part of the weights' gradient both."""
    g = gen(T + C)
    s, w, dy = stream(g, T, C), (1 + 0.3 * randn(g, C)).to(BF), (1e-3 * randn(g, T, C)).to(BF)
    want, E, dw, Ew = backward_ref(dy, s, w, None)
    say(T, C)
    dx, dweight = nv.nvfp4_rms_norm_backward(dy.cuda(), s.cuda(), w.cuda(), eps=EPS)
    assert ((dx.cpu().double() - want).abs() <= E + 2.0 ** -8 * (want.abs() + E) + 1e-38).all()
    assert ((dweight.cpu().double() - dw).abs() <= Ew + U * dw.abs() + 1e-38).all()
    in_place = dy.cuda()
    again = nv.nvfp4_rms_norm_backward(in_place, s.cuda(), w.cuda(), eps=EPS, dx=in_place)
    assert torch.equal(in_place, dx) and torch.equal(again[1], dweight)
