"""Attention over the paged cache where its weights are small: a long tail behind tokens that hold nearly all of the sum, pages whose
scales say little about their values.

Bounds (u = 2^-24), for weights w relative to the row's largest and W their sum:
 weights   2^-11 w (two f16 numbers for fp32 output: 2^-22 w), and no less than 2^-30, each times its own token's |v|: what f16 holds
           (2^-25 at least) where the running maximum stands at 2^7 or more and a page's scale takes up to two binades of it; 2^-31
           where all pages have the scale one, an exponent that takes none.
 scores    a relative error E of every weight, numerator and denominator: 2 E A, A = sum w |v| / W.  Scores that are exact
           sums: 5 u |x| for the factor and the product (x = s log2(e)), u (|x| + 16) for what is added in the exponent, 2 u for the exponential:
           below (8 |s| + 16) u.  Others as in test_kv_attention: (d + 16) u (scale sum |q k| + 8) + 4 u |s|.
 sums      (n + 8) u A, and the result's rounding: 2^-8 |o| (bf16), 4 u |o| (fp32).
"""
import math

import pytest
import torch

import paper_2605_18739_amd as nv
from tests.test_kv_attention import BF, CHUNKS, DECODE, F32, U, attention_case, gen, held, run_attention, say

pytestmark = pytest.mark.gpu


def check_weights(got, q, c, table, lens, starts, scale, causal, out_f32, exact_scores=False, least=2.0 ** -30, window=0, sink=0):
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
        if window:
            see &= (j[None] > p[:, None] - window) | (j[None] < sink)
        for h in range(q.shape[1]):
            qh, kh, va = q[i0:i0 + rows, h].cpu().double(), k[:, h // G], v[:, h // G].abs()
            s = (qh @ kh.T * scale).masked_fill(~see, -math.inf)
            E = (8 * s.abs() + 16) * U if exact_scores else (d + 16) * U * (qh.abs() @ kh.abs().T * scale + 8) + 4 * U * s.abs()
            E = E.masked_fill(~see, 0.0).amax(-1, keepdim=True)
            some = see.any(-1, keepdim=True)
            w = torch.exp(s - torch.where(some, s.amax(-1, keepdim=True), 0.0))
            W = w.sum(-1, keepdim=True).clamp(min=1e-300)
            o, A = w @ v[:, h // G] / W, w @ va / W
            lost = torch.where(see, (w * 2.0 ** (-22 if out_f32 else -11)).clamp(min=least), 0.0) @ va / W
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
        check_weights(out, q, c, table, [n], [0, queries], float(torch.tensor(scale, dtype=F32)), False, out_f32, exact_scores=True, least=2.0 ** -31)

@pytest.mark.parametrize("out_f32", [False, True])
def test_weights_of_ordinary_caches(out_f32):
    for causal, cases in ((True, [(lens, [1] * len(lens), *rest) for lens, *rest in DECODE]), (True, CHUNKS), (False, CHUNKS)):
        for lens, queries, Hq, H, d, page, smooth, what in cases:
            say("[precision] ordinary", what, causal, out_f32)
            c, table, starts, q = attention_case(61, lens, queries, Hq, H, d, page, smooth, gain=2.0)
            out, _ = run_attention(c, table, lens, starts, q, max(queries), causal, out_f32=out_f32, check=False)
            check_weights(out, q, c, table, lens, starts, d ** -0.5, causal, out_f32)

# ---------------------------------------------------------------------------------------------------------------------
# page scales
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("queries", [1, 40])
@pytest.mark.parametrize("out_f32", [False, True])
@pytest.mark.parametrize("d,page,smooth", [(64, 16, False), (80, 48, False), (128, 64, True), (128, 16, True), (256, 32, False)])
@pytest.mark.parametrize("scale", [1e-5, 2e-7, 2e-8, 1e-15])
def test_pages_of_zeros_with_a_scale_of_one(queries, out_f32, d, page, smooth, scale):
    """A page of zeros, whose scale the chunk quantizers set to one, first, last or in between: the others keep their digits."""
    say("[precision] zeros", queries, out_f32, d, page, smooth, scale)
    lens = [page, 3 * page, 7 * page + 5, 700]
    c, table, starts, q = attention_case(62, lens, [queries] * 4, 4, 2, d, page, smooth)
    c.v_global.copy_(scale * (0.3 + torch.rand(c.n_pages, generator=gen(63))))
    for b, zero in enumerate(([], [0], [2, 5], [1, 3, (700 - 1) // page])):
        for p in zero:
            c.v_codes[table[b, p]], c.v_global[table[b, p]] = 0, 1.0
    out, _ = run_attention(c, table, lens, starts, q, queries, False, out_f32=out_f32, check=False)
    check_weights(out, q, c, table, lens, starts, d ** -0.5, False, out_f32)


@pytest.mark.parametrize("queries", [1, 4, 40, 150])
@pytest.mark.parametrize("out_f32", [False, True])
@pytest.mark.parametrize("d,page", [(64, 16), (80, 16), (128, 16), (128, 32), (128, 80), (256, 16)])
def test_page_scales_of_all_magnitudes(queries, out_f32, d, page):
    """Scales up to 2^60 apart, from page to page, and what a page holds does not go by its scale."""
    say("[precision] magnitudes", queries, out_f32, d, page)
    lens = [900, 150, 16]
    c, table, starts, q = attention_case(64, lens, [min(queries, n) for n in lens], 4, 2, d, page, False)
    g = gen(65)
    c.v_global.copy_(2.0 ** (60 * torch.rand(c.n_pages, generator=g) - 30))
    c.v_scales[torch.rand(c.n_pages, generator=g) < 0.5] = 0
    for causal, window, sink in ((True, 0, 0), (False, 0, 0), (True, 100, 20)):
        out, lse = run_attention(c, table, lens, starts, q, queries, causal, window=window, sink=sink, out_f32=out_f32, check=False)
        check_weights(out, q, c, table, lens, starts, d ** -0.5, causal, out_f32, window=window, sink=sink)
        again, lse_again = run_attention(c, table, lens, starts, q, queries, causal, window=window, sink=sink, out_f32=out_f32, check=False)
        assert torch.equal(out, again) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("queries,d", [(1, 128), (5, 64), (40, 64), (40, 256), (200, 128)])
def test_page_scales_of_all_magnitudes_in_pieces(queries, d):
    """The same over a cache that is cut into pieces, whose units differ."""
    say("[precision] magnitudes in pieces", queries, d)
    c, table, starts, q = attention_case(69, [6000], [queries], 2, 1, d, 16, False)
    g = gen(70)
    c.v_global.copy_(2.0 ** (60 * torch.rand(c.n_pages, generator=g) - 30))
    c.v_scales[torch.rand(c.n_pages, generator=g) < 0.5] = 0
    for out_f32 in (False, True):
        out, _ = run_attention(c, table, [6000], starts, q, queries, True, out_f32=out_f32, check=False)
        check_weights(out, q, c, table, [6000], starts, d ** -0.5, True, out_f32)


@pytest.mark.parametrize("queries", [1, 40])
def test_scales_at_the_ends_of_the_range(queries):
    """Results near the largest and the smallest numbers, whole and joined from pieces."""
    say("[precision] ends", queries)
    for exponent in (104, -84):
        for n in (150, 6000):
            c, table, starts, q = attention_case(66, [n], [queries], 2, 1, 64, 16, False)
            c.v_global.copy_(2.0 ** exponent * (0.5 + torch.rand(c.n_pages, generator=gen(67))))
            out, _ = run_attention(c, table, [n], starts, q, queries, False, out_f32=True, check=False)
            check_weights(out, q, c, table, [n], starts, 0.125, False, True)

@pytest.mark.parametrize("queries", [1, 40])
@pytest.mark.parametrize("smooth", [False, True])
def test_the_largest_queries(queries, smooth):
    """Queries up to the largest bf16 number, the keys' scales (and means) as small: the results of 2^-125 times the queries."""
    say("[precision] largest", queries, smooth)
    gain, scale = 2.0 ** 125, 2.0 ** -9
    c, table, starts, q = attention_case(68, [100, 20], [queries] * 2, 4, 2, 64, 16, smooth, gain=64.0)
    q = q.clamp(-7.96875, 7.96875)
    q[0, 0, 0] = 7.96875
    want = run_attention(c, table, [100, 20], starts, q, queries, True, out_f32=True, scale=scale)
    c.k_global.mul_(1 / gain)
    if smooth:
        c.k_mean.copy_((c.k_mean.double() / gain).to(BF))
    big = (q.double() * gain).to(BF)
    assert torch.isfinite(big.float()).all() and float(big.abs().max()) > 2.0 ** 127
    got = run_attention(c, table, [100, 20], starts, big, queries, True, out_f32=True, scale=scale)
    n = starts[-1]
    if not smooth:                                                  # (the same digits; means and their quotients may round apart)
        assert torch.equal(got[0][:n], want[0][:n])


@pytest.mark.parametrize("n", [40, 900, 6000])
@pytest.mark.parametrize("queries,d", [(1, 64), (1, 128), (5, 256), (40, 64), (200, 128), (40, 256)])
def test_the_sum_counts_pages_of_every_scale(queries, d, n):
    """Value scales over the whole range of normal numbers (below 2^126), page by page: each token is in the sum with its weight.  The scores are
    zero, so the sum is the number of tokens: 8 u for a token's weight (its exponent, of up to 2^8, within u 2^8: 2^8 u), (n + 8) u for the sum."""
    say("[precision] sums", queries, d, n)
    g = gen(71)
    for low, high in ((-126, 125), (-126, -90), (100, 125)):
        c = bare_cache(-(-n // 16), 16, 1, d)
        c.v_scales.zero_()
        scales = (1 + torch.rand(c.n_pages, generator=g, dtype=torch.float64)) * 2.0 ** torch.randint(low, high + 1, (c.n_pages,), generator=g).double()
        c.v_global.copy_(scales.to(F32))
        table = torch.arange(c.n_pages, dtype=torch.int32).view(1, -1)
        out, lse = run_attention(c, table, [n], [0, queries], torch.ones((queries, 2, d), dtype=BF), queries, False, out_f32=True, check=False)
        assert (out == 0).all()
        assert float((lse.double() - math.log(n)).abs().max()) <= (2 ** 8 + n + 16) * U + 4 * U * math.log(n), (low, high)


def test_the_sum_of_millions_of_tokens_on_pages_of_the_least_scales():
    """2^22 tokens with equal weights: lanes add up to 2^16 of them, (2^16 + 2^8 + 16) u."""
    n = 1 << 22
    c = bare_cache(n // 4096, 4096, 1, 16)
    c.v_codes.fill_(0x22)
    c.v_scales.fill_(0x38)
    table = torch.arange(c.n_pages, dtype=torch.int32).view(1, -1)
    for exponent in (-126, -100, -90, 0, 110):
        say("[precision] millions", exponent)
        c.v_global.fill_(2.0 ** exponent)
        out, lse = run_attention(c, table, [n], [0, 1], torch.ones((1, 1, 16), dtype=BF), 1, False, out_f32=True, check=False)
        assert float((lse.double() - math.log(n)).abs().max()) <= (2 ** 16 + 2 ** 8 + 16) * U
        if exponent >= -84:
            assert float((out.double() * 2.0 ** -exponent - 1).abs().max()) <= (2 ** 17 + 2 ** 8 + 16) * U + 2.0 ** -22


@pytest.mark.parametrize("queries", [1, 40, 150])
@pytest.mark.parametrize("smooth", [False, True])
def test_scores_that_are_too_small_for_a_number(queries, smooth):
    """Queries and key scales whose products vanish: equal weights for what a row sees, masked tokens left out."""
    for softmax_scale in (0.125, 1e-40):
        say("[precision] vanishing", queries, smooth, softmax_scale)
        c, table, starts, q = attention_case(72, [200, 75], [min(queries, 75)] * 2, 4, 2, 64, 16, smooth)
        c.k_global.fill_(2.0 ** -100)
        if smooth:
            c.k_mean.zero_()
        q = (q.sign() * 2.0 ** -120).to(BF)
        for causal, window in ((True, 0), (True, 37), (False, 0)):
            run_attention(c, table, [200, 75], starts, q, queries, causal, window=window, out_f32=True, scale=softmax_scale)
