"""Calls that read what the call right before them wrote, over and over in the same memory with other values each time: every kernel may be resident while the
one before it still runs, and none may read before that one is over."""
import pytest
import torch

from paper_2605_16732_b200 import binding as dq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,K", [(64, 64), (300, 512), (4096, 3000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", [dq.LAYOUT_NK, dq.LAYOUT_KN])
def test_quantize_and_dequantize(rows, K, dtype, layout):
    g = torch.Generator(device="cuda").manual_seed(rows)
    inputs = [torch.randn((rows, K), device="cuda", generator=g).to(dtype) * 4 ** i for i in range(4)]
    first, second = dq.dirotq_mxfp4_alloc(rows, K), dq.dirotq_mxfp4_alloc(*((rows, K) if layout == dq.LAYOUT_NK else (K, rows)))
    x, out = torch.zeros((rows, K), dtype=dtype, device="cuda"), torch.zeros((second.rows, second.K), dtype=torch.bfloat16, device="cuda")

    def chain(v, wait):
        for step in (lambda: dq.dirotq_mxfp4_quantize(v, out=first), lambda: dq.dirotq_mxfp4_dequantize(first, x),
                     lambda: dq.dirotq_mxfp4_quantize(x, out=second, layout=layout), lambda: dq.dirotq_mxfp4_dequantize(second, out)):
            step()
            if wait:
                torch.cuda.synchronize()

    want = []
    for v in inputs:
        chain(v, True)
        want.append(out.clone())
    for i in range(24):
        chain(inputs[i % 4], False)
        assert torch.equal(out, want[i % 4]), i


@pytest.mark.parametrize("M", [2, 40, 700])
def test_linear_norm_and_linear(M):
    """A block's front: q/k/v of tokens that a linear has just made, then the norm in place and the next linear on the q of it."""
    K, hq, hk, D = 512, 4, 2, 128
    N, g = (hq + 2 * hk) * D, torch.Generator(device="cuda").manual_seed(M)
    w0, w1, w2 = (dq.dirotq_mxfp4_quantize(torch.randn(s, device="cuda", generator=g) * 0.05) for s in ((K, K), (N, K), (K, hq * D)))
    inputs = [torch.randn((M, K), device="cuda", generator=g).bfloat16() * 3 ** i for i in range(3)]
    angle = torch.rand((M, D // 2), device="cuda", generator=g) * 6
    qk, ws = dq.QkNorm(hq, hk, D, rope="halves", cos=angle.cos(), sin=angle.sin()), dq.alloc_mxfp4_workspace(M, max(K, hq * D))
    a, y, z = (torch.zeros((M, n), dtype=torch.bfloat16, device="cuda") for n in (K, N, K))

    def chain(v, wait):
        for step in (lambda: dq.dirotq_mxfp4_linear(v, w0, a, ws), lambda: dq.dirotq_mxfp4_linear(a, w1, y, ws),
                     lambda: dq.dirotq_qk_norm_rope(y, qk, y[:, :hq * D], y[:, hq * D:(hq + hk) * D]), lambda: dq.dirotq_mxfp4_linear(y[:, :hq * D], w2, z, ws),
                     lambda: dq.dirotq_mxfp4_linear(z, w0, a, ws)):
            step()
            if wait:
                torch.cuda.synchronize()

    want = []
    for v in inputs:
        chain(v, True)
        want.append([t.clone() for t in (a, y, z)])
    for i in range(24):
        chain(inputs[i % 3], False)
        assert all(torch.equal(o, t) for o, t in zip((a, y, z), want[i % 3])), i
    assert dq.dirotq_workspace_status(ws) == 0
