"""Descriptions of queries and keys as a C caller may hold them: fields that a call has no use for are left over from another call."""
import ctypes

import pytest
import torch

from paper_2605_16732_b200 import binding as dq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,D", [(3, 64), (60, 128), (300, 64)])
def test_positions_of_another_call_where_nothing_is_rotated(M, D):
    """Positions of a shorter call, all of them out of range, and a table of no rows: with no rotation they say nothing."""
    hq, hk, K = 4, 2, 320
    width = (hq + 2 * hk) * D
    g = torch.Generator(device="cuda").manual_seed(M)
    w_q, w_k = (1 + 0.3 * torch.randn((2, D), device="cuda", generator=g)).bfloat16()
    plan, stale = (dq.QkNorm(hq, hk, D, q_weight=w_q, k_weight=w_k) for _ in range(2))
    left_over = torch.full((4096,), -1, dtype=torch.int32, device="cuda")  # (long enough for every token: nothing here can be read out of range)
    stale.struct.positions = left_over.data_ptr()
    assert stale.struct.rope == 0 and ctypes.sizeof(stale.struct) == ctypes.sizeof(plan.struct)
    x = torch.randn((M, K), device="cuda", generator=g).bfloat16()
    w = dq.dirotq_mxfp4_quantize(torch.randn((width, K), device="cuda", generator=g) * 0.1)
    ws = dq.alloc_mxfp4_workspace(M, K)
    fused, apart = [], []
    for p in (plan, stale):
        y = torch.empty((M, width), dtype=torch.bfloat16, device="cuda")
        dq.dirotq_mxfp4_qkv(x, w, y, ws, p)
        fused.append(y)
        q, k = torch.empty((M, hq * D), dtype=torch.bfloat16, device="cuda"), torch.empty((M, hk * D), dtype=torch.bfloat16, device="cuda")
        dq.dirotq_qk_norm_rope(y, p, q, k)
        apart.append(torch.cat((q, k), 1))
    assert dq.dirotq_workspace_status(ws) == 0
    assert torch.equal(fused[0], fused[1]) and torch.equal(apart[0], apart[1])
