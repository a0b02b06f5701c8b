"""Norm / rotation, the paged NVFP4 cache and attention over it as a program uses them: one after another, captured, on other
streams, with pages that are not in use, far slots and many sequences.  Bounds as in test_kv_attention; where two runs do
the same arithmetic, bit for bit."""
import math

import pytest
import torch

import paper_2605_18739_amd as nv
from tests.test_kv_attention import (BF, F32, attention_case, attention_ref, check_slots, fill_cache, gen, new_cache, norm_ref, randn, rope_inputs, rotation,
                                     run_attention, say, U)

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def clone_cache(c):
    return nv.NVFP4KvCache(k_codes=c.k_codes.clone(), k_scales=c.k_scales.clone(), k_global=c.k_global.clone(), v_codes=c.v_codes.clone(), v_scales=c.v_scales.clone(),
                           v_global=c.v_global.clone(), k_mean=None if c.k_mean is None else c.k_mean.clone())


# ---------------------------------------------------------------------------------------------------------------------
# the operators together
# ---------------------------------------------------------------------------------------------------------------------
class Model:
    """The attention of one layer: queries, keys and values side by side in one row of a fused projection."""

    def __init__(self, seed, Hq, H, d, page, pages, smooth, axes=3):
        self.g, self.Hq, self.H, self.d, self.page = gen(seed), Hq, H, d, page
        self.cache = new_cache(pages, page, H, d, smooth, seed)
        self.wq, self.wk = ((1 + 0.2 * randn(self.g, d)).to(BF).cuda() for _ in range(2))
        _, self.freqs, self.parts = rope_inputs(self.g, 1, d // 2, axes, 100)
        self.freqs_there = self.freqs.cuda()

    def project(self, T):
        return randn(self.g, T, self.Hq + 2 * self.H, self.d).to(BF).cuda()

    def step(self, qkv, positions, slots, table, lens, starts, max_q, causal, out=None, lse=None, workspace=None, **kw):
        Hq, H = self.Hq, self.H
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        qr, kr = nv.nvfp4_qk_norm_rope(q, k, self.wq, self.wk, nv.NVFP4Rope(positions, self.freqs_there, self.parts, True))
        nv.nvfp4_kv_cache_write(self.cache, kr, v, slots)
        out, lse = nv.nvfp4_kv_attention(qr, self.cache, table, lens, starts, max_q, causal=causal, out=out, lse=lse, workspace=workspace, **kw)
        return qr, kr, v, out, lse


@pytest.mark.parametrize("smooth", [False, True])
@pytest.mark.parametrize("Hq,H,d", [(4, 4, 128), (8, 2, 64)])
def test_prompt_then_single_tokens(oracle, Hq, H, d, smooth):
    say("[use] prompt then tokens", Hq, H, d, smooth)
    page, lens = 16, [37, 5, 64]
    m = Model(31, Hq, H, d, page, 20, smooth)
    table = torch.randperm(20, generator=m.g)[:18].reshape(3, 6).to(torch.int32)
    where = lambda b, j: int(table[b, j // page]) * page + j % page
    for turn in range(5):                                  # the prompt, then a token of each sequence at a time
        new = lens if turn == 0 else [1] * 3
        now = lens if turn == 0 else [n + turn for n in lens]
        T = sum(new)
        starts = [0, new[0], new[0] + new[1], T]
        at = [(b, now[b] - new[b] + i) for b in range(3) for i in range(new[b])]
        positions = torch.tensor([[j, j // 7, j % 7] for _, j in at], dtype=torch.int32)
        slots = torch.tensor([where(b, j) for b, j in at])
        qkv = m.project(T)
        before = clone_cache(m.cache)
        qr, kr, v, out, lse = m.step(qkv, positions.cuda(), slots.cuda(), table.cuda(), ints(now), ints(starts), max(new), True)
        torch.cuda.synchronize()
        R = rotation(positions, m.freqs, m.parts, d, True)
        for x, w, got in ((qkv[:, :Hq], m.wq, qr), (qkv[:, Hq:Hq + H], m.wk, kr)):
            want, mag = norm_ref(x.cpu(), w.cpu(), R, 1e-6)
            assert ((got.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 32 * U * mag).all()
        alone = new_cache(20, page, H, d, smooth, 31)
        nv.nvfp4_kv_cache_write(alone, kr, v, slots.cuda())
        check_slots(oracle, alone, kr, v, slots, False, "step")
        for a, b in zip(m.cache._native, alone._native):
            if a is not None and a.dim() > 1:
                assert torch.equal(a.flatten(0, 1)[slots.cuda()], b.flatten(0, 1)[slots.cuda()])
        rest = torch.ones(20 * page, dtype=torch.bool)
        rest[slots] = False
        assert torch.equal(m.cache.k_codes.cpu().flatten(0, 1)[rest], before.k_codes.cpu().flatten(0, 1)[rest]), "slots of other tokens"
        want, want_lse, bo, bl = attention_ref(qr, m.cache, table, now, starts, max(new), d ** -0.5, True, 0, 0, False)
        assert ((out.cpu().double() - want).abs() <= bo).all() and ((lse.cpu().double() - want_lse).abs() <= bl).all()


def test_a_chunk_sees_pages_that_the_chunk_quantizers_filled():
    Hq = H = 3
    d, page = 128, 48
    say("[use] quantized chunks")
    c = nv.NVFP4KvCache.empty(4, page, H, d, smooth=True)
    g = gen(32)
    k, v = (randn(g, 4, page, H, d) + 0.5).to(BF).cuda(), randn(g, 4, page, H, d).to(BF).cuda()
    for p in range(4):
        kd, mean, vd = c.page(p)
        nv.nvfp4_kv_quant_k(k[p], out=kd, row_mean=mean)
        nv.nvfp4_kv_quant(v[p], out=vd)
    q = randn(g, page, Hq, d).to(BF)
    run_attention(c, torch.tensor([[2, 0, 3, 1]], dtype=torch.int32), [4 * page], [0, page], q, page, False)


# ---------------------------------------------------------------------------------------------------------------------
# graphs, streams
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("queries", [1, 40])
def test_captured_steps_follow_lengths_and_pages(queries):
    """Two graphs of the same step that share a workspace, replayed in turn with eager work between them."""
    say("[use] graphs", queries)
    B, page, pages = 3, 16, 600
    m = Model(33, 8, 2, 64, page, pages, True, axes=1)
    T = B * queries
    starts = ints([queries * b for b in range(B + 1)])
    n = nv.nvfp4_kv_attention_workspace_bytes(T, 8, 2, 64, 180 * page, B, queries)
    assert n > 0
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    static = dict(qkv=m.project(T), positions=torch.zeros((T, 1), dtype=torch.int32, device="cuda"), slots=torch.full((T,), -1, dtype=torch.int64, device="cuda"),
                  table=torch.zeros((B, 180), dtype=torch.int32, device="cuda"), lens=ints([queries] * B))
    outs = [(torch.empty((T, 8, 64), dtype=BF, device="cuda"), torch.empty((T, 8), dtype=F32, device="cuda")) for _ in range(2)]
    fill_cache(m.cache, m.g)

    def step(o):
        return m.step(static["qkv"], static["positions"], static["slots"], static["table"], static["lens"], starts, queries, True, out=o[0], lse=o[1], workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in outs:
            step(o)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(o)
        graphs.append(g)
    for turn in range(6):
        lens = [queries + int(x) for x in torch.randint(0, 180 * page - queries, (B,), generator=m.g)]
        if turn == 3:
            lens[1] = queries
        table = torch.randperm(pages, generator=m.g)[:B * 180].reshape(B, 180).to(torch.int32)
        at = [(b, lens[b] - queries + i) for b in range(B) for i in range(queries)]
        static["qkv"].copy_(m.project(T))
        static["positions"].copy_(torch.tensor([[j] for _, j in at], dtype=torch.int32))
        static["slots"].copy_(torch.tensor([int(table[b, j // page]) * page + j % page for b, j in at]))
        static["table"].copy_(table)
        static["lens"].copy_(ints(lens))
        for o in outs:
            o[0].fill_(7.0), o[1].fill_(7.0)
        for g in graphs if turn % 2 else graphs[::-1]:
            g.replay()
        ws.fill_(255)                                      # (nothing in it survives a call)
        want = m.step(static["qkv"], static["positions"], static["slots"], static["table"], static["lens"], starts, queries, True)
        torch.cuda.synchronize()
        for o in outs:
            assert same(o[0], want[3]) and same(o[1], want[4]), turn
        graphs[turn % 2].replay()                          # after eager work and a synchronisation
        torch.cuda.synchronize()
        assert same(outs[turn % 2][0], want[3])


def test_captured_backward_of_the_norm():
    say("[use] backward in a graph")
    g = gen(34)
    T, Hq, H, d = 50, 4, 2, 64
    positions, freqs, parts = rope_inputs(g, T, 32, 2, 100)
    rope = nv.NVFP4Rope(positions.cuda(), freqs.cuda(), parts, True)
    make = lambda h: randn(g, T, h, d).to(BF).cuda()
    w = [(1 + 0.2 * randn(g, d)).to(BF).cuda() for _ in range(2)]
    static = [make(Hq), make(H), make(Hq), make(H)]
    run = lambda: nv.nvfp4_qk_norm_rope_backward(*static, *w, rope)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for turn in range(4):
        for t in static:
            t.copy_(randn(g, *t.shape).to(BF))
        graph.replay()
        want = run()
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(captured, want)), turn


def test_on_other_streams_at_once():
    say("[use] streams")
    cases = [attention_case(35 + s, [3000, 50, 700], [1, 1, 1], 8, 2, 128, 16, True) for s in range(2)]
    args = [(c, table.cuda(), ints([3000, 50, 700]), ints(starts), q.cuda()) for c, table, starts, q in cases]
    call = lambda a, out, **kw: nv.nvfp4_kv_attention(a[4], a[0], a[1], a[2], a[3], 1, causal=True, out=out, **kw)
    outs = [[torch.zeros(a[4].shape, dtype=BF, device="cuda") for _ in range(9)] for a in args]
    want = [call(a, o[8]) for a, o in zip(args, outs)]
    k = randn(gen(40), 3, 2, 128).to(BF).cuda()
    slots = torch.tensor([5, 700, 31], device="cuda")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for n in range(8):
        for a, o, s, r in zip(args, outs, streams, got):
            r.append(call(a, o[n], stream=s))
    back = nv.nvfp4_kv_cache_read(args[0][0], slots, stream=streams[0])
    torch.cuda.synchronize()
    for w, runs in zip(want, got):
        for r in runs:
            assert same(r[0][:3], w[0][:3]) and same(r[1][:3], w[1][:3])
    assert all(same(a, b) for a, b in zip(back, nv.nvfp4_kv_cache_read(args[0][0], slots)))
    nv.nvfp4_kv_cache_write(args[0][0], k, k, slots, stream=streams[1])
    streams[1].synchronize()
    other = clone_cache(args[0][0])
    nv.nvfp4_kv_cache_write(other, k, k, slots)
    torch.cuda.synchronize()
    assert torch.equal(other.k_codes, args[0][0].k_codes) and torch.equal(other.v_scales, args[0][0].v_scales)


# ---------------------------------------------------------------------------------------------------------------------
# pages
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("queries", [1, 30])
@pytest.mark.parametrize("d", [64, 80, 128, 256])
@pytest.mark.parametrize("bad", [0.0, -2.0, math.inf, math.nan, 1e-40])
def test_pages_that_are_not_in_use(queries, d, bad):
    """Ids outside the pool, and pages behind the window or the length, whatever their scales and bytes are."""
    say("[use] unused pages", queries, d, bad)
    H, Hq, page, window, sink = 2, 4, 16, 90, 20
    smooth = d != 80
    lens = [230, 40]
    c, table, starts, q = attention_case(41, lens, [queries] * 2, Hq, H, d, page, smooth)
    used = {int(p) for row in table for p in row if p >= 0}
    spare = [p for p in range(c.n_pages) if p not in used]
    # tokens 32 .. 95: behind the sink of 20, and before the window of the first query, which sees 111 on (queries 200 .. 229)
    table[0, 2:6] = torch.tensor([spare[0], c.n_pages, -(1 << 31), (1 << 31) - 1])
    table[1, 3:] = torch.tensor([spare[1]] * (table.shape[1] - 3))                      # behind the length of 40
    # page 0, which stands in for ids outside the pool, is one of the pages not in use
    swap = spare[0]
    moved = lambda t: torch.where(t == 0, swap, torch.where(t == swap, 0, t)).to(torch.int32)
    table = moved(table)
    order = list(range(c.n_pages))
    order[0], order[swap] = swap, 0
    c = nv.NVFP4KvCache(*(t if t is None else t[order].contiguous() for t in (c.k_codes, c.k_scales, c.k_global, c.v_codes, c.v_scales, c.v_global, c.k_mean)))
    clean, unused = clone_cache(c), [0, swap if spare[1] == 0 else spare[1]]
    for p in unused:
        for t in (c.k_global, c.v_global):
            t[p] = bad
        for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales):
            t[p] = 255
        if smooth:
            c.k_mean[p] = math.nan
        for t in (clean.k_global, clean.v_global):
            t[p] = 1.0
    got = run_attention(c, table, lens, starts, q, queries, True, window=window, sink=sink, check=False)
    want = run_attention(clean, table, lens, starts, q, queries, True, window=window, sink=sink)
    assert same(got[0], want[0]) and same(got[1], want[1])
    assert torch.isfinite(got[0].float()).all()


@pytest.mark.parametrize("queries", [1, 5, 70])
def test_ids_outside_the_pool_are_not_seen(queries):
    say("[use] ids outside", queries)
    c, table, starts, q = attention_case(42, [200, 90], [queries] * 2, 4, 2, 64, 16, True)
    table[0, 2], table[0, 5], table[0, 11] = -1, c.n_pages, 1 << 30
    table[1, :] = -7                                       # a sequence that sees nothing at all
    run_attention(c, table, [200, 90], starts, q, queries, True)
    run_attention(c, table, [200, 90], starts, q, queries, False)


@pytest.mark.parametrize("queries", [1, 24])
def test_sequences_that_share_pages(queries):
    say("[use] shared pages", queries)
    c, table, starts, q = attention_case(50, [150, 150, 40], [queries] * 3, 4, 2, 128, 16, True)
    table[1] = table[0]
    table[2, :2] = table[0, 0]                             # and a sequence that holds one page twice
    run_attention(c, table, [150, 133, 40], starts, q, queries, True)
    run_attention(c, table, [150, 133, 40], starts, q, queries, False, window=50, sink=3)


def test_lengths_and_queries_are_cut_off():
    say("[use] cut off")
    for queries in ([1, 1], [3, 20], [60, 30]):
        c, table, starts, q = attention_case(43, [100, 64], queries, 4, 2, 64, 16, False)
        run_attention(c, table, [100000, 1 << 30], starts, q, max(queries), False)        # as far as the table goes (whose -1 are not seen)
        got, want = (run_attention(c, table, [n, 64], starts, q, max(queries), True, check=n == 0) for n in (-5, 0))
        assert same(got[0], want[0]) and same(got[1], want[1])
        run_attention(c, table, [100, 64], starts, q, max(1, max(queries) // 2), True)    # queries from max_q on are not computed
        many = torch.cat([table, torch.full((2, 300), -1, dtype=torch.int32)], 1)         # a table for far longer caches
        run_attention(c, many, [100, 64], starts, q, max(queries), True)


def test_slots_past_32_bits_of_every_plane():
    """Pages whose codes lie past 4 GiB and whose row number times head size passes 2^32."""
    H, d, page, pages = 8, 128, 1024, 9000
    say("[use] far slots", pages * page * H * d // 2 / 2 ** 30, "GiB of codes")
    far = nv.NVFP4KvCache.empty(pages, page, H, d, smooth=True)
    small = nv.NVFP4KvCache.empty(4, page, H, d, smooth=True)
    ids = [8999, 8750, 3, 8998]
    for c, pp in ((far, ids), (small, range(4))):
        for n, p in enumerate(pp):
            c.k_global[p], c.v_global[p] = 0.01 * (n + 1), 0.02
    g = gen(44)
    T = 2600
    k, v = randn(g, T, H, d).to(BF).cuda(), randn(g, T, H, d).to(BF).cuda()
    j = torch.arange(T)
    at = lambda pp: (torch.tensor(pp)[j // page] * page + j % page).cuda()
    for c, pp in ((far, ids), (small, list(range(4)))):
        nv.nvfp4_kv_cache_write(c, k, v, at(pp))
    a, b = nv.nvfp4_kv_cache_read(far, at(ids)), nv.nvfp4_kv_cache_read(small, at(list(range(4))))
    assert all(same(x, y) for x, y in zip(a, b))
    for queries in (1, 50):
        q = randn(g, queries, 16, d).to(BF).cuda()
        r = [nv.nvfp4_kv_attention(q, c, ints([list(pp)]), ints([T]), ints([0, queries]), queries, causal=True) for c, pp in ((far, ids), (small, range(4)))]
        torch.cuda.synchronize()
        assert same(r[0][0], r[1][0]) and same(r[0][1], r[1][1])
    del far
    torch.cuda.empty_cache()


def test_many_sequences():
    """More sequences than lanes, of very different lengths: pieces of all of them lie one behind the other."""
    say("[use] 150 sequences")
    lens = [(b * 7) % 40 for b in range(150)]
    lens[3], lens[70], lens[149] = 2500, 900, 1600
    c, table, starts, q = attention_case(45, lens, [1] * 150, 2, 1, 64, 16, True)
    run_attention(c, table, lens, starts, q, 1, True)
    queries = [b % 3 for b in range(150)]                  # some without any
    starts = [sum(queries[:b]) for b in range(151)]
    run_attention(c, table, lens, starts, q[:starts[-1] + 2], 2, True, out_f32=True)


def test_more_blocks_of_rows_than_the_chip_holds():
    say("[use] 528 blocks of rows, the last 16 in pieces")
    B, H, queries = 33, 8, 140
    lens = [1100 if b == 32 else 150 for b in range(B)]
    c, table, starts, q = attention_case(46, lens, [queries] * B, H, H, 16, 16, False)
    run_attention(c, table, lens, starts, q, queries, True, out_f32=True)


# ---------------------------------------------------------------------------------------------------------------------
# strides and magnitudes
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("queries", [1, 33])
@pytest.mark.parametrize("out_f32", [False, True])
def test_queries_and_results_inside_wider_rows(queries, out_f32):
    say("[use] strides", queries, out_f32)
    c, table, starts, q = attention_case(47, [100, 20], [queries] * 2, 4, 2, 64, 16, True)
    want = run_attention(c, table, [100, 20], starts, q, queries, True, out_f32=out_f32)
    wide = torch.full((q.shape[0], 7, 64), math.nan, dtype=BF, device="cuda")
    wide[:, 2:6] = q.cuda()
    out = torch.full((q.shape[0], 9, 64), 3.0, dtype=F32 if out_f32 else BF, device="cuda")
    nv.nvfp4_kv_attention(wide[:, 2:6], c, table.cuda(), ints([100, 20]), ints(starts), queries, causal=True, out_dtype=nv.OUT_F32 if out_f32 else nv.OUT_BF16, out=out[:, 4:8])
    torch.cuda.synchronize()
    assert same(out[:, 4:8].contiguous(), want[0])
    assert (out[:, :4] == 3.0).all() and (out[:, 8:] == 3.0).all()


@pytest.mark.parametrize("queries", [1, 33])
@pytest.mark.parametrize("gain", [2.0 ** 100, 2.0 ** -100])
def test_magnitudes_of_queries_and_of_page_scales(queries, gain):
    """Powers of two move from the queries to the keys' scales and to the values' without a change in the results' digits."""
    say("[use] magnitudes", queries, gain)
    c, table, starts, q = attention_case(48, [100, 20], [queries] * 2, 4, 2, 64, 16, False)
    want = run_attention(c, table, [100, 20], starts, q, queries, True)
    n = starts[-1]
    other = clone_cache(c)
    other.k_global.mul_(1 / gain)
    got = run_attention(other, table, [100, 20], starts, (q.double() * gain).to(BF), queries, True)
    assert same(got[0][:n], want[0][:n])
    other = clone_cache(c)
    other.v_global.mul_(2.0 ** 60 if gain > 1 else 2.0 ** -60)
    run_attention(other, table, [100, 20], starts, q, queries, True)


@pytest.mark.parametrize("queries", [1, 20])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_query_that_is_not_finite_spoils_its_own_row_alone(queries, bad):
    say("[use] not finite", queries, bad)
    c, table, starts, q = attention_case(49, [100, 20], [queries] * 2, 4, 2, 64, 16, True)
    want, want_lse, bo, bl = attention_ref(q, c, table, [100, 20], starts, queries, 64 ** -0.5, True, 0, 0, False)
    q[queries - 1, 1, 5] = bad
    out, lse = run_attention(c, table, [100, 20], starts, q, queries, True, check=False)
    keep = ~torch.isnan(want_lse) & ~torch.isinf(want_lse)
    keep[queries - 1, 1] = False
    assert ((out.cpu().double() - want).abs() <= bo)[keep].all() and ((lse.cpu().double() - want_lse).abs() <= bl)[keep].all()
    assert not torch.isfinite(out[queries - 1, 1].float()).all()

@pytest.mark.parametrize("queries", [1, 20])
@pytest.mark.parametrize("tokens", [20, 3000])
def test_a_row_without_a_number_says_so(queries, tokens):
    """A query whose scores are no numbers: its result and its log of the sum are NaN (-inf is for rows that see nothing)."""
    say("[use] lse of NaN", queries, tokens)
    c, table, starts, q = attention_case(51, [tokens, 100, 0], [queries] * 3, 4, 2, 64, 16, True)
    q[queries - 1, 1, 5] = math.nan
    q[2 * queries - 1, 3] = math.inf                                # (inf - inf in every score with keys of both signs)
    out, lse = run_attention(c, table, [tokens, 100, 0], starts, q, queries, False, check=False)
    for row, head in ((queries - 1, 1), (2 * queries - 1, 3)):
        assert torch.isnan(out[row, head].float()).all() and torch.isnan(lse[row, head])
    rest = torch.ones(lse[:3 * queries].shape, dtype=torch.bool)
    rest[queries - 1, 1] = rest[2 * queries - 1, 3] = False
    assert not torch.isnan(lse[:3 * queries].cpu()[rest]).any()
    assert (lse[2 * queries:3 * queries] == -math.inf).all() and (out[2 * queries:3 * queries] == 0).all()

@pytest.mark.parametrize("interleaved,pairs", [(True, 21), (True, 8), (False, 8), (False, 16)])
def test_elements_that_are_not_turned_stay_as_they_are(interleaved, pairs):
    """Infinities, NaN and signed zeros from 2 P on, in values and in gradients: neither they nor their neighbours change."""
    say("[norm_rope] not turned", interleaved, pairs)
    g = gen(71)
    T, H, d = 9, 5, 64
    x = randn(g, T, H, d).to(BF)
    rest = x[..., 2 * pairs:]
    for n, special in enumerate((math.inf, -math.inf, math.nan, -0.0)):
        rest[..., n::7] = special
    positions = torch.randint(1, 5000, (T, 1), generator=g, dtype=torch.int32)
    freqs = torch.rand(pairs, generator=g)
    rope = nv.NVFP4Rope(positions.cuda(), freqs.cuda(), [pairs], interleaved)
    clean = x.clone()
    clean[..., 2 * pairs:] = 0
    bits = lambda t: t.cpu().contiguous().view(torch.int16)
    for run in (lambda t: nv.nvfp4_qk_norm_rope(t.cuda(), None, None, None, rope)[0], lambda t: nv.nvfp4_qk_norm_rope_backward(t.cuda(), None, None, None, None, None, rope)[0]):
        y, turned = run(x), run(clean)
        assert torch.equal(bits(y[..., 2 * pairs:]), bits(x[..., 2 * pairs:]))
        assert torch.equal(bits(y[..., :2 * pairs]), bits(turned[..., :2 * pairs]))

# ---------------------------------------------------------------------------------------------------------------------
# outputs that the calls allocate
# ---------------------------------------------------------------------------------------------------------------------
def leave_garbage(*sizes):
    """Freed blocks of these sizes, full of 0xFF: what a new output finds."""
    blocks = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
    torch.cuda.synchronize()
    del blocks


@pytest.mark.parametrize("d,H", [(64, 3), (80, 24), (256, 1)])
def test_new_outputs_of_a_read_hold_zeros_for_slots_outside_the_cache(d, H):
    say("[use] new outputs of a read", d, H)
    c = nv.NVFP4KvCache.empty(3, 32, H, d)
    fill_cache(c, gen(52))
    slots = torch.randperm(96, generator=gen(53))[:70]
    slots[[0, 5, 33, 69]] = torch.tensor([-1, 96, -(1 << 40), 1 << 40])
    outside = (slots < 0) | (slots >= 96)
    given = [torch.full((70, H, d), 5.0, dtype=BF, device="cuda") for _ in range(2)]
    nv.nvfp4_kv_cache_read(c, slots.cuda(), *given)
    for stream in (None, torch.cuda.Stream()):
        leave_garbage(70 * H * d * 2)
        got = nv.nvfp4_kv_cache_read(c, slots.cuda(), stream=stream)
        torch.cuda.synchronize()
        for x, y in zip(got, given):
            assert same(x[~outside.cuda()], y[~outside.cuda()])
            assert (x[outside.cuda()] == 0).all() and (y[outside.cuda()] == 5.0).all()


@pytest.mark.parametrize("queries", [1, 3, 40])
@pytest.mark.parametrize("out_f32", [False, True])
@pytest.mark.parametrize("long", [False, True])
def test_new_outputs_of_attention_hold_zeros_where_no_sequence_computes(queries, out_f32, long):
    """Rows in front of the first sequence and behind the last one, and queries from max_q on: zeros and -inf."""
    say("[use] new outputs of attention", queries, out_f32, long)
    lens, n = [4000 if long else 100, 30, 0], [queries + 2, queries, queries]
    c, table, starts, q = attention_case(54, lens, n, 4, 2, 64, 16, False)
    table = table.cuda()
    q = torch.cat([q[:3], q, q[:150]]).cuda()                       # rows before and behind
    starts = [3 + s for s in starts]
    computed = torch.zeros(q.shape[0], dtype=torch.bool)
    for b in range(3):
        computed[starts[b]:starts[b] + min(n[b], queries)] = True
    kind = nv.OUT_F32 if out_f32 else nv.OUT_BF16
    given = torch.full(q.shape, 3.0, dtype=F32 if out_f32 else BF, device="cuda"), torch.full(q.shape[:2], 4.0, device="cuda")
    call = lambda **kw: nv.nvfp4_kv_attention(q, c, table, ints(lens), ints(starts), queries, causal=True, out_dtype=kind, **kw)
    call(out=given[0], lse=given[1])
    assert (given[0][~computed.cuda()] == 3.0).all() and (given[1][~computed.cuda()] == 4.0).all()
    leave_garbage(given[0].nbytes, given[1].nbytes)
    fresh = call()
    torch.cuda.synchronize()
    half = call(out=torch.full_like(given[0], 3.0)), call(lse=torch.full_like(given[1], 4.0))
    for out, lse, rest_o, rest_l in ((*fresh, 0.0, -math.inf), (*half[0], 3.0, -math.inf), (*half[1], 0.0, 4.0)):
        assert same(out[computed.cuda()], given[0][computed.cuda()]) and same(lse[computed.cuda()], given[1][computed.cuda()])
        assert (out[~computed.cuda()] == rest_o).all() and (lse[~computed.cuda()] == rest_l).all()
