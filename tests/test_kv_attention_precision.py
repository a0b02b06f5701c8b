"""Attention over the paged cache where its weights are small: a long tail behind tokens that hold nearly all of the sum.

Bounds (u = 2^-24), for weights w relative to the row's largest and W their sum:
 weights   2^-11 w (two f16 numbers for fp32 output: 2^-22 w), and no less than 2^-31, each times its own token's |v|: what f16 holds
           (2^-25 at least) where the running maximum stands at 2^9 or more, and three binades to spare.
 scores    a relative error E of every weight, numerator and denominator: 2 E A, A = sum w |v| / W.  Scores that are exact
           sums: 5 u |x| for the factor and the product (x = s log2(e)), u (|x| + 16) for what is added in the exponent, 2 u for the exponential:
           below (8 |s| + 16) u.  Others as in test_kv_attention: (d + 16) u (scale sum |q k| + 8) + 4 u |s|.
 sums      (n + 8) u A, and the result's rounding: 2^-8 |o| (bf16), 4 u |o| (fp32).
"""
import math

import pytest
import torch

import paper_2605_18739_amd as nv
from tests.test_kv_attention import BF, F32, U, gen, held, run_attention, say

pytestmark = pytest.mark.gpu


def check_weights(got, q, c, table, lens, starts, scale, causal, out_f32, exact_scores=False):
    """out of run_attention against 64 bits, every weight's error with its own token's values."""
    G, page, d, planes = q.shape[1] // c.H, c.page_tokens, c.d, [None if t is None else t.cpu() for t in c._native]
    got, worst = got.cpu().double(), 0.0
    for b, n in enumerate(lens):
        i0, rows = starts[b], starts[b + 1] - starts[b]
        if n == 0 or rows == 0:
            continue
        j = torch.arange(n)
        slots = table[b].long()[j // page] * page + j % page
        k, v = held(planes[0], planes[1], planes[2], planes[3], page, slots), held(planes[4], planes[5], planes[6], None, page, slots)
        p = n - rows + torch.arange(rows) if causal else torch.full((rows,), n - 1)
        see = j[None] <= p[:, None]
        for h in range(q.shape[1]):
            qh, kh, va = q[i0:i0 + rows, h].cpu().double(), k[:, h // G], v[:, h // G].abs()
            s = (qh @ kh.T * scale).masked_fill(~see, -math.inf)
            E = (8 * s.abs() + 16) * U if exact_scores else (d + 16) * U * (qh.abs() @ kh.abs().T * scale + 8) + 4 * U * s.abs()
            E = E.masked_fill(~see, 0.0).amax(-1, keepdim=True)
            some = see.any(-1, keepdim=True)
            w = torch.exp(s - torch.where(some, s.amax(-1, keepdim=True), 0.0))
            W = w.sum(-1, keepdim=True).clamp(min=1e-300)
            o, A = w @ v[:, h // G] / W, w @ va / W
            lost = torch.where(see, (w * 2.0 ** (-22 if out_f32 else -11)).clamp(min=2.0 ** -31), 0.0) @ va / W
            bound = (4 * U if out_f32 else 2.0 ** -8) * o.abs() + lost + (2 * E + (n + 8) * U) * A
            err = (got[i0:i0 + rows, h] - o).abs()
            worst = max(worst, float((err / bound.clamp(min=1e-300)).max()))
    assert worst <= 1.0, worst


def bare_cache(pages, page, H, d):
    """Keys of zero, values of random codes at block scales of 1 to 1.875, tensor scales of one."""
    g = gen(pages)
    c = nv.NVFP4KvCache.empty(pages, page, H, d)
    c.v_codes.copy_(torch.randint(0, 256, c.v_codes.shape, generator=g, dtype=torch.uint8))
    c.v_scales.copy_(torch.randint(0x38, 0x40, c.v_scales.shape, generator=g, dtype=torch.uint8))
    c.k_scales.fill_(0x38)
    return c


@pytest.mark.parametrize("queries", [1, 40])
@pytest.mark.parametrize("out_f32", [False, True])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n", [300, 5000])
def test_a_long_tail_behind_dominant_tokens(queries, out_f32, d, n):
    """Every sixteenth token's values are zero and its score lies `below` binades above all others, whose values are the result
    (every sixteenth: whatever piece of the tokens a wave takes)."""
    page = 64
    c = bare_cache(80, page, 1, d)
    c.k_codes[:, ::16], c.v_codes[:, ::16] = 0x22, 0                # (keys of ones)
    table = torch.arange(80, dtype=torch.int32).view(1, 80)
    for below in (12.3, 18.7, 24.6):
        say("[precision] tail", queries, out_f32, d, n, below)
        q = torch.ones((queries + 2, 2, d), dtype=BF)
        q[:, 1] = 0.9375                                            # (the other head's distance is a sixteenth less)
        scale = below * math.log(2) / d
        out, _ = run_attention(c, table, [n], [0, queries], q, queries, False, scale=scale, out_f32=out_f32, check=False)
        check_weights(out, q, c, table, [n], [0, queries], float(torch.tensor(scale, dtype=F32)), False, out_f32, exact_scores=True)
