"""Quantized values against the elements they stand for, and operands made on another stream in memory that was just handed back."""
import pytest
import torch

import mx_reference as ref
from paper_2605_16732_b200 import binding as dq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rule", [ref.FLOOR, ref.CEIL])
@pytest.mark.parametrize("layout", [dq.LAYOUT_NK, dq.LAYOUT_KN])
def test_values_within_half_a_step(rule, layout):
    """Of an element u times the block's scale: levels are 1/2 apart up to 2, 1 up to 4, 2 up to 6, so the value is off by at most half of that; above 6
    (at most 8, and only with the specification's rule) it is 6.  Scales are powers of two and values have two bits: exact in 64 bits, no slack."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn((200, 333), generator=g) * torch.exp2(torch.randint(-100, 100, (200, 1), generator=g).float())
    x[3], x[4, :40], x[5, ::3] = 0, -0.0, 1e-42
    t = dq.dirotq_mxfp4_quantize((x if layout == dq.LAYOUT_NK else x.T.contiguous()).cuda(), scale_rule=rule, layout=layout)
    y = torch.empty((200, 333), device="cuda")
    dq.dirotq_mxfp4_dequantize(t, y)
    _, scales = dq.dirotq_mxfp4_export(t)
    s = torch.exp2(scales.cpu().double() - 127).repeat_interleave(32, 1)[:, :333]
    u, v = x.double().abs() / s, y.cpu().double() / s * torch.where(x < 0, -1.0, 1.0)
    assert float(u.max()) < 8 and (rule == ref.FLOOR or float(u.max()) <= 6)
    half = torch.where(u <= 2, 0.25, torch.where(u <= 4, 0.5, 1.0))
    assert bool(((u - v).abs() <= half)[u <= 6].all()) and bool((v == 6)[u > 6].all())
    # blocks of normal numbers use the upper half of the levels: the largest element is above 3 scales (CEIL), or at least 4 (FLOOR)
    top = torch.nn.functional.pad(u, (0, -333 % 32)).unflatten(1, (-1, 32)).amax(2)
    normal = scales.cpu() > 0
    assert bool(((top > 3) if rule == ref.CEIL else (top >= 4))[normal].all()) and int(normal.sum()) > 1500


@pytest.mark.parametrize("how", ["quantize", "import"])
def test_operands_made_on_another_stream_in_memory_still_to_be_written(how):
    """The memory of an operand given back while the current stream is still to fill it is handed out again: what is made there on another stream comes after."""
    rows, K = 300, 4096
    x = torch.randn((rows, K), generator=torch.Generator().manual_seed(1)).bfloat16()
    codes, scales = ref.quantize(x)
    xd, packed, scales_d = x.cuda(), ref.pack(codes).cuda(), scales.cuda()  # (uploaded before: a copy from pageable memory would wait for the fill)
    side = torch.cuda.Stream()

    def make():
        return dq.dirotq_mxfp4_quantize(xd, stream=side) if how == "quantize" else dq.dirotq_mxfp4_import(packed, scales_d, K, stream=side)

    make().buffer.fill_(0)  # (a kernel's first launch may wait for the device)
    torch.cuda._sleep(1000)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    old = dq.dirotq_mxfp4_alloc(rows, K)
    torch.cuda.synchronize()
    busy = torch.cuda.Event()
    torch.cuda._sleep(40_000_000)
    old.buffer.fill_(255)
    busy.record()
    where = old.buffer.data_ptr()
    old.close()
    del old
    t = make()
    still_busy = not busy.query()
    torch.cuda.synchronize()
    assert t.buffer.data_ptr() == where and still_busy  # (else nothing was tested)
    got, got_scales = dq.dirotq_mxfp4_export(t)
    assert torch.equal(ref.unpack(got.cpu(), K), codes) and torch.equal(got_scales.cpu(), scales)
