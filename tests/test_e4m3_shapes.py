"""Every kernel that the rule of the 8-bit products can choose, over several turns of its loop.  Bounds: tests/test_e4m3.py.

tests/test_e4m3_plan.py checks on the CPU that the sizes below reach every kernel.
"""
import pytest
import torch

import paper_2605_18739_amd as nv
from tests.test_e4m3 import BF, E8M0, U, act_ref, assert_codes, gen, poisoned, say, small_integers, values

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
