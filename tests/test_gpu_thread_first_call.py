"""A call that is the first thing its thread does on the GPU (buffers, layers and operands come from another one): on a thread the device's context is not current
until a call makes it so, and the tensor maps that a call encodes need it."""
import ctypes
import threading

import pytest
import torch

from paper_2605_16732_b200 import binding as dq

pytestmark = pytest.mark.gpu


def _on_a_new_thread(call):
    errors = []

    def work():
        try:
            call()
        except BaseException as e:  # (to be seen by the test)
            errors.append(e)

    torch.cuda.synchronize()
    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not errors, errors


@pytest.mark.parametrize("M", [3, 64, 300])  # (3: quantized by the product's own blocks, no tensor map made)
@pytest.mark.parametrize("name", ["linear", "qkv"])
def test_mxfp4(M, name):
    K, hq, hk, D = 512, 4, 1, 64
    N = (hq + 2 * hk) * D
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randn((M, K), device="cuda", generator=g).bfloat16()
    w, ws, qk = dq.dirotq_mxfp4_quantize(torch.randn((N, K), device="cuda", generator=g)), dq.alloc_mxfp4_workspace(M, K), dq.QkNorm(hq, hk, D)
    want, y = (torch.zeros((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def call(out):
        if name == "linear":
            dq.dirotq_mxfp4_linear(x, w, out, ws)
        else:
            dq.dirotq_mxfp4_qkv(x, w, out, ws, qk)

    _on_a_new_thread(lambda: call(y))
    call(want)
    assert torch.equal(y, want) and dq.dirotq_workspace_status(ws) == 0


def test_operands_are_made():
    """dirotq_mxfp4_create encodes the operand's own maps."""
    n = dq.dirotq_mxfp4_bytes(300, 256)
    buffer = dq._alloc_bytes(n, "cuda")
    handle = ctypes.c_void_p(0)
    _on_a_new_thread(lambda: dq._check(dq.lib().dirotq_mxfp4_create(300, 256, buffer.data_ptr(), n, ctypes.byref(handle)), "dirotq_mxfp4_create"))
    assert handle.value
    dq._check(dq.lib().dirotq_mxfp4_destroy(handle), "dirotq_mxfp4_destroy")


@pytest.mark.parametrize("fmt", ["int4", "int4_asym", "w4a8", "nvfp4", "int4_ph", "nvfp4_ph"])
@pytest.mark.parametrize("M", [16, 300])
def test_prepared_layers(fmt, M):
    from test_gpu_qkv_forms import _prepared
    K, N = 512, 384
    g = torch.Generator(device="cuda").manual_seed(M)
    Q = torch.linalg.qr(torch.randn((K, K), dtype=torch.float64, device="cuda", generator=g))[0].contiguous()
    layer = _prepared(fmt, 0.05 * torch.randn((K, N), device="cuda", generator=g), Q)
    x, ws = torch.randn((M, K), device="cuda", generator=g).bfloat16(), dq.alloc_workspace(layer, M)
    want, y = (torch.zeros((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    _on_a_new_thread(lambda: dq.dirotq_linear(x, layer, y, ws))
    dq.dirotq_linear(x, layer, want, ws)
    assert torch.equal(y, want) and dq.dirotq_workspace_status(ws) == 0
    layer.close()
