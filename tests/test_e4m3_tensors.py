"""An E4M3Tensor whose tensors change after it was made: calls take what it holds then, and refuse what no longer fits together."""
import pytest
import torch

import paper_2605_18739_amd as nv
from tests.test_e4m3 import BF, E4M3, E8M0, gen, randn, raw, values


def test_sizes_follow_what_is_held():
    codes, scales = torch.zeros((256, 512), dtype=E4M3), torch.zeros((256, 4), dtype=torch.uint8).view(E8M0)
    t = nv.E4M3Tensor(codes, scales)
    t.codes, t.scales = torch.zeros((300, 272), dtype=E4M3), torch.zeros((3, 3), dtype=torch.uint8).view(E8M0)
    assert (t.rows, t.K, t.block_rows) == (300, 272, 128)
    c = t.c()
    assert (c.codes, c.scales, c.rows, c.K, c.block_rows) == (t.codes.data_ptr(), t.scales.data_ptr(), 300, 272, 128)


def pair(seed, M=70, N=256, K=512):
    g = gen(seed)
    return nv.nvfp4_e4m3_quantize(randn(g, M, K).to(BF).cuda()), nv.nvfp4_e4m3_quantize_2d(randn(g, N, K).to(BF).cuda(), transposed=False)[0]


@pytest.mark.gpu
def test_operands_that_were_assigned():
    """Weights replaced in a tensor that a program holds: the product, and the gated one, are those of the new ones."""
    (A, W), (B, V) = pair(1), pair(2)
    want, want_h = nv.nvfp4_e4m3_gemm(B, V), nv.nvfp4_e4m3_gemm_gated(B, V)[0]
    assert not torch.equal(nv.nvfp4_e4m3_gemm(A, W), want)
    A.codes, A.scales, W.codes, W.scales = B.codes, B.scales, V.codes, V.scales
    assert torch.equal(nv.nvfp4_e4m3_gemm(A, W), want)
    assert all(torch.equal(x, y) for x, y in zip(raw(nv.nvfp4_e4m3_gemm_gated(A, W)[0]), raw(want_h)))
    assert torch.equal(values(A), values(B))
    # fewer rows, and scales by rows instead of by tiles
    A.codes, A.scales = B.codes[:33], B.scales[:33]
    W.scales = V.scales.view(torch.uint8).repeat_interleave(128, 0).view(E8M0)
    assert torch.equal(nv.nvfp4_e4m3_gemm(A, W), nv.nvfp4_e4m3_gemm(nv.E4M3Tensor(B.codes[:33], B.scales[:33]), V))


@pytest.mark.gpu
def test_outputs_that_were_assigned():
    """Results go to what the tensor holds at the time of the call; what it held before stays as it is."""
    x = randn(gen(3), 128, 256).to(BF).cuda()
    want = nv.nvfp4_e4m3_quantize(x)
    out = nv.E4M3Tensor.empty(128, 256)
    old = out.codes.view(torch.uint8).fill_(0xEE), out.scales.view(torch.uint8).fill_(0xEE)
    out.codes, out.scales = torch.empty_like(out.codes), torch.empty_like(out.scales)
    assert nv.nvfp4_e4m3_quantize(x, out=out) is out
    assert all(torch.equal(p, q) for p, q in zip(raw(out), raw(want))) and all((o == 0xEE).all() for o in old)


@pytest.mark.gpu
def test_tensors_that_no_longer_fit_are_refused():
    x = randn(gen(4), 128, 256).to(BF).cuda()

    def changed(change):
        t = nv.nvfp4_e4m3_quantize(x)
        change(t)
        return t
    W = nv.nvfp4_e4m3_quantize_2d(x, transposed=False)[0]
    for change in (lambda t: t.codes.t_(), lambda t: t.scales.t_(), lambda t: t.codes.resize_(64, 256), lambda t: t.codes.resize_(256, 256), lambda t: t.codes.resize_(128, 512),
                   lambda t: t.scales.resize_(128, 1), lambda t: setattr(t, "codes", t.codes.float()), lambda t: setattr(t, "scales", t.scales.float()),
                   lambda t: setattr(t, "codes", t.codes[:, ::2]), lambda t: setattr(t, "scales", t.scales[:64]), lambda t: setattr(t, "codes", t.codes.cpu()),
                   lambda t: setattr(t, "codes", t.codes[0])):
        for call in (lambda: nv.nvfp4_e4m3_gemm(changed(change), W), lambda: nv.nvfp4_e4m3_gemm(W, changed(change)), lambda: nv.nvfp4_e4m3_quantize(x, out=changed(change)),
                     lambda: nv.nvfp4_rms_norm(x, torch.ones(256, dtype=BF, device="cuda"), out=changed(change))):
            with pytest.raises(AssertionError):
                call()
    for bad in (None, (1, 2), 3):
        with pytest.raises(TypeError):
            nv.nvfp4_e4m3_gemm(changed(lambda t: setattr(t, "scales", bad)), W)
