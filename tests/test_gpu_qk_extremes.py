"""Norm and rotation of q and k at the ends of the range that the header gives: the sum of squares is held in fp32."""
import pytest
import torch

from paper_2605_16732_b200 import binding as dq
from test_gpu_qk_norm import Setup, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,rot,style", [(256, 256, "halves"), (128, 128, "pairs"), (72, 36, "halves"), (128, 48, "halves"), (64, 0, None)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("largest", [1e18, 1e-17])
def test_largest_and_smallest_heads(D, rot, style, dtype, largest):
    """Without eps the scale of a head drops out: up to 1e18 the squares of 256 elements add up below fp32's largest number, from 1e-17 on their mean is a normal
    number, and what the smaller ones lose as subnormal numbers is below 2^-149 of 1e-34 each."""
    s = Setup(9, 5, 3, D, rot, style, dtype, D, eps=0.0)
    heads = torch.randn((9, 11, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    heads = heads / heads.abs().amax(-1, keepdim=True) * (largest * (1 - 2.0 ** -6 if largest > 1 else 1 + 2.0 ** -6))  # (inside the range after rounding to 8 bits)
    heads[0] = largest * (1 - 2.0 ** -6 if largest > 1 else 1 + 2.0 ** -6)  # every element of a head
    heads[1, :, 1:] = 0                                                    # only one
    x = heads.flatten(1).to(dtype)
    q, k = (torch.empty((9, n * D), dtype=dtype, device="cuda") for n in (5, 3))
    dq.dirotq_qk_norm_rope(x, s.plan, q, k)
    (wq, tq), (wk, tk), _ = s.want(x)
    _within(q, wq, tq)
    _within(k, wk, tk)


def test_heads_of_zeros():
    for eps in (0.0, 1e-6):
        s = Setup(3, 2, 1, 64, 64, "pairs", torch.bfloat16, 1, eps=eps)
        x = torch.zeros_like(s.x)
        q, k = (torch.empty((3, n * 64), dtype=torch.bfloat16, device="cuda") for n in (2, 1))
        dq.dirotq_qk_norm_rope(x, s.plan, q, k)
        assert bool((torch.isnan(q) if eps == 0 else q == 0).all()) and bool((torch.isnan(k) if eps == 0 else k == 0).all())
