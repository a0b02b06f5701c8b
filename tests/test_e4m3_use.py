"""The feed-forward half of a block in 8 bits as a program uses it: forward and backward in a row, captured into graphs, on other
streams, with large tensors; and what the calls refuse.

The chain is compared step by step: each step's inputs are read back, and its outputs have to be what the step's definition in 64
bits makes of them, within the bounds of tests/test_e4m3.py and tests/test_rms_norm.py.
"""
import math

import pytest
import torch

import paper_2605_18739_amd as nv
from tests.test_e4m3 import BF, E4M3, E8M0, F32, F64, U, act_ref, assert_codes, assert_exact, ceil, gen, quantized, randn, raw, say, values
from tests.test_rms_norm import backward_ref, norm_ref, slack

pytestmark = pytest.mark.gpu


class Block:
    """Norm of the residual stream, gated projections and down projection with weights in 8 bits."""

    def __init__(self, C, F, seed):
        g = gen(seed)
        self.norm = (1 + 0.2 * randn(g, C)).to(BF).cuda()
        self.w_gate_up, self.w_down = (randn(g, 2 * F, C) / math.sqrt(C)).to(BF).cuda(), (randn(g, C, F) / math.sqrt(F)).to(BF).cuda()
        self.gu, self.gu_t = nv.nvfp4_e4m3_quantize_2d(self.w_gate_up)
        self.down, self.down_t = nv.nvfp4_e4m3_quantize_2d(self.w_down)

    def forward(self, x, residual):
        a, y, s = nv.nvfp4_rms_norm(x, self.norm, residual, keep_bf16=True)
        h, _, gate_up = nv.nvfp4_e4m3_gemm_gated(a, self.gu, keep_gate_up=True)
        out = nv.nvfp4_e4m3_gemm(h, self.down, out_dtype=nv.OUT_BF16)
        return out, (a, y, s, h, gate_up)

    def backward(self, dout, dsum, kept):
        a, y, s, h, gate_up = kept
        d = nv.nvfp4_e4m3_quantize(dout)
        dh = nv.nvfp4_e4m3_gemm(d, self.down_t, out_dtype=nv.OUT_BF16)
        dgu, dgu_t, h_t, _ = nv.nvfp4_gated_backward(dh, gate_up, recompute_h=True)
        dy = nv.nvfp4_e4m3_gemm(dgu, self.gu_t, out_dtype=nv.OUT_BF16)
        d_t, y_t = nv.nvfp4_e4m3_quantize(dout, block_axis=1), nv.nvfp4_e4m3_quantize(y, block_axis=1)
        dw_down, dw_gu = nv.nvfp4_e4m3_gemm(d_t, h_t), nv.nvfp4_e4m3_gemm(dgu_t, y_t)
        dx, dnorm = nv.nvfp4_rms_norm_backward(dy, s, self.norm, dsum)
        return dx, dnorm, dw_gu, dw_down, (d, dh, dgu, dgu_t, h_t, dy, d_t, y_t)


def inputs(T, C, seed):
    g = gen(seed)
    return randn(g, T, C).to(BF).cuda(), (3 * randn(g, T, C)).to(BF).cuda(), (0.1 * randn(g, T, C)).to(BF).cuda(), (0.1 * randn(g, T, C)).to(BF).cuda()


def assert_product(y, A, W, what):
    a, w = values(A), values(W)
    want, S = a @ w.T, a.abs() @ w.abs().T
    E = a.shape[1] * 2 * U * S
    E = E + 2.0 ** -8 * (want.abs() + E) if y.dtype == BF else E
    assert ((y.cpu().double() - want).abs() <= E).all(), what


@pytest.mark.parametrize("T,C,F", [(1, 256, 384), (16, 400, 256), (65, 512, 640), (333, 640, 1152)])
def test_block_forward_and_backward(T, C, F):
    b = Block(C, F, T)
    x, r, dout, dsum = inputs(T, C, T + 1)
    say(T, C, F)
    out, kept = b.forward(x, r)
    a, y, s, h, gate_up = kept
    dx, dnorm, dw_gu, dw_down, steps = b.backward(dout, dsum, kept)
    d, dh, dgu, dgu_t, h_t, dy, d_t, y_t = steps
    # forward
    assert torch.equal(s.cpu(), (x.float() + r.float()).to(BF).cpu())
    want = norm_ref(s.cpu(), b.norm.cpu())
    assert_codes(a, want, slack(C) * want.abs(), "norm")
    va, vw = values(a), values(b.gu)
    gu, E = va @ vw.T, C * 2 * U * (va.abs() @ vw.abs().T)
    act, up = act_ref(nv.ACT_SILU, gu[:, :F])[0], gu[:, F:]
    Eh = up.abs() * (1.13 * E[:, :F] + 8 * U * (gu[:, :F].abs() + 1) * act.abs()) + act.abs() * E[:, F:] + 4 * U * (act * up).abs() + 1.13 * E[:, :F] * E[:, F:]
    assert_codes(h, act * up, Eh, "h")
    assert_product(out, h, b.down, "out")
    # backward
    assert_exact(d, quantized(dout.cpu().double()), "dout")
    assert_product(dh, d, b.down_t, "dh")
    vdh, vg, vu = dh.cpu().double(), gate_up[:, :F].cpu().double(), gate_up[:, F:].cpu().double()
    act, slope = act_ref(nv.ACT_SILU, vg)
    want = torch.cat([vdh * vu * slope, vdh * act], 1)
    E = 32 * U * torch.cat([(vdh * vu).abs(), (vdh * act).abs()], 1) * (1 + vg.abs()).repeat(1, 2) + 1e-38
    assert_codes(dgu, want, E, "gated backward")
    T16 = 16 * ceil(T, 16)

    def turned(v):
        o = torch.zeros((v.shape[1], T16), dtype=F64)
        o[:, :T] = v.T
        return o
    assert_codes(dgu_t, turned(want), turned(E), "gated backward, along the tokens")
    assert_product(dy, dgu, b.gu_t, "dy")
    assert_exact(y_t, quantized(turned(y.cpu().double())), "y along the tokens")
    assert_product(dw_down, d_t, h_t, "dw_down")
    assert_product(dw_gu, dgu_t, y_t, "dw_gu")
    want, E, dw, Ew = backward_ref(dy.cpu(), s.cpu(), b.norm.cpu(), dsum.cpu())
    assert ((dx.cpu().double() - want).abs() <= E + 2.0 ** -8 * (want.abs() + E)).all()
    assert ((dnorm.cpu().double() - dw).abs() <= Ew + U * dw.abs()).all()


def test_gradients_of_the_block_point_the_same_way():
    """Against the gradients of the unquantized block (fp32 autograd): every tensor passes at most five roundings to 8 bits on the way,
    each within 2^-4 of each element and independent of the others' signs: the relative error stays below 5 * 2^-4 of the norm."""
    T, C, F = 256, 512, 768
    b = Block(C, F, 3)
    x, r, dout, dsum = inputs(T, C, 4)
    out, kept = b.forward(x, r)
    dx, dnorm, dw_gu, dw_down, _ = b.backward(dout, dsum, kept)
    s = kept[2].float().requires_grad_()
    norm, wg, wd = (w.float().requires_grad_() for w in (b.norm, b.w_gate_up, b.w_down))
    y = s * torch.rsqrt(s.square().mean(1, keepdim=True) + 1e-6) * norm
    gu = y @ wg.T
    ref = (torch.nn.functional.silu(gu[:, :F]) * gu[:, F:]) @ wd.T
    (ref * dout.float()).sum().backward()
    for name, got, want in (("out", out, ref.detach()), ("dx", dx, s.grad + dsum.float()), ("dnorm", dnorm, norm.grad), ("dw_gu", dw_gu, wg.grad), ("dw_down", dw_down, wd.grad)):
        off = float((got.float() - want).norm() / want.norm())
        say(name, off)
        assert off <= 5 * 2.0 ** -4, name


def flat(v):
    for t in v:
        if isinstance(t, nv.E4M3Tensor):
            yield t.codes.view(torch.uint8)
            yield t.scales.view(torch.uint8)
        elif isinstance(t, torch.Tensor):
            yield t.view(torch.uint8) if t.dtype in (E4M3, E8M0) else t
        elif isinstance(t, tuple):
            yield from flat(t)


@pytest.mark.parametrize("T", [5, 200])
def test_captured_and_replayed(T):
    """Forward and backward captured once, replayed over new contents of the same buffers with eager runs in between."""
    C, F = 512, 640
    b = Block(C, F, 7)
    buffers = inputs(T, C, 8)

    def step():
        out, kept = b.forward(buffers[0], buffers[1])
        return out, kept, b.backward(buffers[2], buffers[3], kept)
    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            captured = step()
    torch.cuda.synchronize()
    for n in range(4):
        for buffer, new in zip(buffers, inputs(T, C, 20 + n)):
            buffer.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in flat(captured)]
        eager = step()
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(got, flat(eager))):
            assert torch.equal(x, y), f"replay {n}, output {i}"


def test_two_graphs_share_a_workspace():
    """Calls that keep their results in buffers of their own may share a workspace as long as they follow each other on a stream."""
    g = gen(1)
    A, W = [nv.nvfp4_e4m3_quantize(randn(g, 9, 512).to(BF).cuda()) for _ in range(2)], nv.nvfp4_e4m3_quantize_2d(randn(g, 512, 512).to(BF).cuda())[0]
    want = [nv.nvfp4_e4m3_gemm_gated(a, W)[0] for a in A]
    ws = torch.empty(nv.nvfp4_workspace_bytes(nv.OP_E4M3_GEMM_GATED, 9, 256), dtype=torch.uint8, device="cuda")
    outs, graphs, side = [nv.E4M3Tensor.empty(9, 256) for _ in A], [], torch.cuda.Stream()
    for a, o in zip(A, outs):
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            nv.nvfp4_e4m3_gemm_gated(a, W, out=o, workspace=ws)
    for n in range(3):
        for o in outs:
            o.codes.view(torch.uint8).fill_(0xEE)
        torch.cuda.synchronize()
        for k in (0, 1, 0):
            graphs[k].replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(raw(o), raw(w)))


def test_other_streams():
    """Every call on a stream of its own gives what it gives on the current one."""
    C, F, T = 512, 640, 70
    b = Block(C, F, 9)
    x, r, dout, dsum = inputs(T, C, 10)
    out, kept = b.forward(x, r)
    a, y, s, h, gate_up = kept
    dh = dout.new_empty((T, F)).normal_().to(BF)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    calls = [lambda **k: nv.nvfp4_rms_norm(x, b.norm, r, keep_bf16=True, **k), lambda **k: nv.nvfp4_e4m3_quantize(x, **k), lambda **k: nv.nvfp4_e4m3_quantize(x, block_axis=1, **k),
             lambda **k: nv.nvfp4_e4m3_quantize_2d(b.w_down, **k), lambda **k: nv.nvfp4_e4m3_gemm(h, b.down, **k), lambda **k: nv.nvfp4_e4m3_gemm(h, b.down, fast_sums=True, **k),
             lambda **k: nv.nvfp4_e4m3_gemm_gated(a, b.gu, keep_h=True, keep_gate_up=True, **k), lambda **k: nv.nvfp4_gated_backward(dh, gate_up, recompute_h=True, keep_bf16=True, **k),
             lambda **k: nv.nvfp4_rms_norm_backward(dout, s, b.norm, dsum, **k)]
    for i, call in enumerate(calls):
        here = call()
        torch.cuda.synchronize()
        there = call(stream=side)
        side.synchronize()
        here, there = (v if isinstance(v, tuple) else (v,) for v in (here, there))
        for p, q in zip(flat(here), flat(there)):
            assert torch.equal(p, q), f"call {i}"


def test_two_calls_at_once():
    """The same operands multiplied on two streams at the same time, into buffers of their own."""
    g = gen(11)
    A, W = nv.nvfp4_e4m3_quantize(randn(g, 600, 2048).to(BF).cuda()), nv.nvfp4_e4m3_quantize_2d(randn(g, 2048, 2048).to(BF).cuda())[0]
    want = nv.nvfp4_e4m3_gemm_gated(A, W)[0]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for n in range(6):
        with torch.cuda.stream(streams[n % 2]):
            got.append(nv.nvfp4_e4m3_gemm_gated(A, W)[0])
    torch.cuda.synchronize()
    for q in got:
        assert all(torch.equal(x, y) for x, y in zip(raw(q), raw(want)))


def test_offsets_past_32_bits():
    """Operands of more than 2^32 elements and results of more than 2^32 bytes: the last rows are what they are on their own."""
    R, C = 270000, 16384
    x = torch.empty((R, C), dtype=BF, device="cuda").normal_()
    q = nv.nvfp4_e4m3_quantize(x)
    tail = nv.nvfp4_e4m3_quantize(x[-300:])
    assert torch.equal(q.codes.view(torch.uint8)[-300:], tail.codes.view(torch.uint8)) and torch.equal(q.scales.view(torch.uint8)[-300:], tail.scales.view(torch.uint8))
    t = nv.nvfp4_e4m3_quantize(x, block_axis=1)
    part = nv.nvfp4_e4m3_quantize(x[:, -64:], block_axis=1)
    assert torch.equal(t.codes.view(torch.uint8)[-64:], part.codes.view(torch.uint8)) and torch.equal(t.scales.view(torch.uint8)[-64:], part.scales.view(torch.uint8))
    del t, part
    w = nv.nvfp4_e4m3_quantize_2d(torch.empty((8208, C), dtype=BF, device="cuda").normal_(), transposed=False)[0]
    y = nv.nvfp4_e4m3_gemm(q, w, out_dtype=nv.OUT_BF16, fast_sums=True)
    assert torch.equal(y[-300:], nv.nvfp4_e4m3_gemm(tail, w, out_dtype=nv.OUT_BF16, fast_sums=True))
    del y, q, w
    n, s = nv.nvfp4_rms_norm(x, torch.ones(C, dtype=BF, device="cuda"), x, keep_bf16=True)[1:]
    m, u = nv.nvfp4_rms_norm(x[-9:], torch.ones(C, dtype=BF, device="cuda"), x[-9:], keep_bf16=True)[1:]
    assert torch.equal(n[-9:], m) and torch.equal(s[-9:], u)
    torch.cuda.synchronize()


def test_not_finite_gated_backward():
    """A NaN or infinity of one token and feature reaches its own blocks and no others."""
    g = gen(12)
    T, F = 300, 256
    dh, gu = randn(g, T, F).to(BF), randn(g, T, 2 * F).to(BF)
    clean = nv.nvfp4_gated_backward(dh.cuda(), gu.cuda(), recompute_h=True)
    dh[130, 5] = math.nan
    bad = nv.nvfp4_gated_backward(dh.cuda(), gu.cuda(), recompute_h=True)
    s, c = raw(bad[0])[1], raw(clean[0])[1]
    assert (s[130, 0] == 255) and (s[130, 2] == 255) and int((s != c).sum()) == 2
    s, c = raw(bad[1])[1], raw(clean[1])[1]
    assert (s[5, 1] == 255) and (s[F + 5, 1] == 255) and int((s != c).sum()) == 2
    assert all(torch.equal(x, y) for x, y in zip(raw(bad[2]), raw(clean[2])))
    assert int(torch.isnan(values(bad[0])).sum()) == 256 and int(torch.isnan(values(bad[1])).sum()) == 256


def test_extreme_scales_of_few_rows():
    """Arrays of scales shorter than a word, and scales over the whole range, for few rows as for many."""
    for M, N, K in ((1, 1, 16), (1, 16, 128), (1, 3, 256), (3, 2, 128), (2, 130, 272)):
        g = gen(M + N + K)
        a, w = randn(g, M, K).to(BF).cuda(), randn(g, N, K).to(BF).cuda()
        for rows_w in ((1, 128) if N % 16 == 0 else (1,)):
            A, W = nv.nvfp4_e4m3_quantize(a), nv.nvfp4_e4m3_quantize(w) if rows_w == 1 else nv.nvfp4_e4m3_quantize_2d(w, transposed=False)[0]
            assert_product(nv.nvfp4_e4m3_gemm(A, W), A, W, (M, N, K))


def test_refusals_of_tensors():
    g = gen(13)
    x = randn(g, 32, 256).to(BF).cuda()
    A = nv.nvfp4_e4m3_quantize(x)
    W = nv.nvfp4_e4m3_quantize_2d(randn(g, 64, 256).to(BF).cuda())[0]
    w = torch.ones(256, dtype=BF, device="cuda")
    for call in (lambda: nv.nvfp4_e4m3_quantize(x.float()), lambda: nv.nvfp4_e4m3_quantize(x.T), lambda: nv.nvfp4_e4m3_quantize(x.cpu()), lambda: nv.nvfp4_e4m3_quantize(x[0]),
                 lambda: nv.nvfp4_e4m3_gemm(A, W, Y=torch.empty((32, 63), device="cuda")), lambda: nv.nvfp4_e4m3_gemm(A, W, Y=torch.empty((32, 64), dtype=BF, device="cuda")),
                 lambda: nv.nvfp4_e4m3_gemm(A, W, Y=torch.empty((64, 32), device="cuda").T), lambda: nv.nvfp4_e4m3_gemm(nv.E4M3Tensor(A.codes.cpu(), A.scales.cpu()), W),
                 lambda: nv.nvfp4_gated_backward(x, x), lambda: nv.nvfp4_rms_norm(x, w[:128]), lambda: nv.nvfp4_rms_norm(x, w, x[:16]), lambda: nv.nvfp4_rms_norm(x, w, sum=x),
                 lambda: nv.nvfp4_rms_norm(x, w.float()), lambda: nv.nvfp4_rms_norm_backward(x, x[:, :128], w), lambda: nv.nvfp4_rms_norm_backward(x, x, w, dweight=torch.empty(255, device="cuda")),
                 lambda: nv.nvfp4_e4m3_gemm_gated(A, W, h=torch.empty((32, 31), dtype=BF, device="cuda"))):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: nv.nvfp4_e4m3_gemm(W, W), lambda: nv.nvfp4_e4m3_gemm(A, A, Y=torch.empty((32, 32), device="cuda").expand(32, 32)[:, :32].as_strided((32, 32), (0, 1))),
                 lambda: nv.nvfp4_e4m3_quantize(x[:, :200]), lambda: nv.nvfp4_e4m3_quantize(x[:, 4:20]), lambda: nv.nvfp4_rms_norm(x, w, eps=0.0),
                 lambda: nv.nvfp4_e4m3_gemm_gated(A, W, act=nv.ACT_NONE), lambda: nv.nvfp4_e4m3_gemm_gated(A, W, quantize=False), lambda: nv.nvfp4_rms_norm(x, w, quantize=False),
                 lambda: nv.nvfp4_e4m3_quantize(x, out=nv.E4M3Tensor.empty(32, 128)), lambda: nv.nvfp4_gated_backward(x[:, :128], x, quantize=False)):
        with pytest.raises(nv.NVFP4Error):
            call()
    for bad in (x, None, (A.codes, A.scales)):
        with pytest.raises((TypeError, AttributeError)):
            nv.nvfp4_e4m3_gemm(bad, W)
