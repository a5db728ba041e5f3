"""Outputs of the MXFP4 linear in the memory of its input: the same bits as elsewhere, on both sides of the row count up to which the product's own blocks
quantize x (which they must not do then: one could write y while another still reads x)."""
import pytest
import torch

from paper_2605_16732_b200 import binding as dq

pytestmark = pytest.mark.gpu


def _quantizer_ran_alone(ws):
    """Whether the call's quantizer left its codes in the workspace (zero before), behind the status block."""
    return bool((ws[1024:] != 0).any())


@pytest.mark.parametrize("M,K", [(1, 256), (1, 8192), (2, 3968), (8, 1024), (31, 256), (32, 256), (33, 256), (60, 1024), (300, 512)])
@pytest.mark.parametrize("shift", [0, -1, 1])
def test_linear_over_its_input(M, K, shift):
    """A square layer whose output takes its input's place, or starts a row before or behind it in one scratch buffer."""
    g = torch.Generator(device="cuda").manual_seed(M + K)
    w = dq.dirotq_mxfp4_quantize(torch.randn((K, K), device="cuda", generator=g) * 0.05)
    x = torch.randn((M, K), device="cuda", generator=g).bfloat16()
    want, ws = torch.empty_like(x), dq.alloc_mxfp4_workspace(M, K)
    dq.dirotq_mxfp4_linear(x, w, want, ws)
    few = M * -(-K // 256) <= 32
    assert _quantizer_ran_alone(ws) == (not few)
    for _ in range(3):
        ws.zero_()
        scratch = torch.full((M + 2, K), 7, dtype=torch.bfloat16, device="cuda")
        scratch[1:1 + M] = x
        y = scratch[1 + shift:1 + shift + M]
        dq.dirotq_mxfp4_linear(scratch[1:1 + M], w, y, ws)
        assert torch.equal(y, want)
        assert dq.dirotq_workspace_status(ws) == 0
        assert _quantizer_ran_alone(ws) or (M == 1 and shift != 0)  # (one row behind the other: no shared byte)


@pytest.mark.parametrize("M", [1, 6, 40])
@pytest.mark.parametrize("x_dtype", [torch.float32, torch.bfloat16])
def test_columns_of_one_scratch_row(M, x_dtype):
    """x and y side by side in the rows of one buffer share nothing, and the few-rows form stays; a y that reaches into x's columns does not get it."""
    K, N = 512, 384
    g = torch.Generator(device="cuda").manual_seed(M)
    w = dq.dirotq_mxfp4_quantize(torch.randn((N, K), device="cuda", generator=g) * 0.05)
    x = torch.randn((M, K), device="cuda", generator=g).to(x_dtype)
    want, ws = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), dq.alloc_mxfp4_workspace(M, K)
    dq.dirotq_mxfp4_linear(x, w, want, ws)
    per = x.element_size() // 2  # 16-bit columns an element of x takes
    for first in (0, K * per - 64, K * per):  # y's first 16-bit column
        ws.zero_()
        rows = torch.zeros((M, K * per + N + 16), dtype=torch.bfloat16, device="cuda")
        here = rows.view(x_dtype)[:, :K]
        here.copy_(x)
        y = rows[:, first:first + N]
        dq.dirotq_mxfp4_linear(here, w, y, ws)
        assert torch.equal(y, want), first
        assert _quantizer_ran_alone(ws) == (first < K * per or M * 2 > 32), first


@pytest.mark.parametrize("M", [2, 8, 64])
def test_qkv_over_its_input(M):
    hq, hk, D, K = 4, 2, 64, 512
    g = torch.Generator(device="cuda").manual_seed(M)
    w = dq.dirotq_mxfp4_quantize(torch.randn((K, K), device="cuda", generator=g) * 0.05)
    angle = torch.rand((M, D // 2), device="cuda", generator=g) * 6
    qk = dq.QkNorm(hq, hk, D, rope="pairs", cos=angle.cos(), sin=angle.sin())
    x = torch.randn((M, K), device="cuda", generator=g).half()
    want, ws = torch.empty_like(x), dq.alloc_mxfp4_workspace(M, K)
    dq.dirotq_mxfp4_qkv(x, w, want, ws, qk)
    ws.zero_()
    dq.dirotq_mxfp4_qkv(x, w, x, ws, qk)
    assert torch.equal(x, want) and _quantizer_ran_alone(ws) and dq.dirotq_workspace_status(ws) == 0
