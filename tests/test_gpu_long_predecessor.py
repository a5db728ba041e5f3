"""The MXFP4 products behind a kernel of another program's that lets the next one start at once and then runs for longer than the library's waits may
last: the time it takes is not theirs."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2605_16732_b200 import binding as dq
from paper_2605_16732_b200 import build

pytestmark = pytest.mark.gpu

# One block that ends by the clock (and, whatever the clock says, after so many turns of at least a microsecond's sleep each).
SOURCE = r"""
#include <cuda_runtime.h>
__global__ void long_kernel(unsigned long long ns) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    for (int i = 0; i < 5000000; ++i) {
        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
        if (t - t0 >= ns) break;
        __nanosleep(2000);
    }
}
extern "C" __attribute__((visibility("default"))) int run_long(unsigned long long ns, void* stream) {
    long_kernel<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>(ns);
    return static_cast<int>(cudaGetLastError());
}
"""


@pytest.fixture(scope="module")
def run_long(tmp_path_factory):
    d = tmp_path_factory.mktemp("long")
    src, so = d / "long.cu", d / "long.so"
    src.write_text(SOURCE)
    subprocess.check_call([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O2", "-Xcompiler", "-fPIC", "-shared", "-cudart", "static", str(src),
                           "-o", str(so)])
    lib = ctypes.CDLL(os.fspath(so))
    lib.run_long.argtypes = [ctypes.c_ulonglong, ctypes.c_void_p]

    def run(seconds):
        assert lib.run_long(int(seconds * 1e9), torch.cuda.current_stream().cuda_stream) == 0

    run(1e-6)  # (loads it)
    torch.cuda.synchronize()
    return run


@pytest.fixture
def gemm_tile():
    yield dq.dirotq_set_gemm_tile
    dq.dirotq_set_gemm_tile(0)


@pytest.mark.parametrize("call,M,columns", [("linear", 2, 0), ("linear", 64, 0), ("gemm", 64, 64), ("gemm", 300, 128), ("gemm", 300, 512), ("qkv", 2, 0)])
def test_waits_leave_it_out(run_long, gemm_tile, call, M, columns):
    K, hq, hk, D = 512, 6, 1, 64
    N = (hq + 2 * hk) * D
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randn((M, K), device="cuda", generator=g).bfloat16()
    w = dq.dirotq_mxfp4_quantize(torch.randn((N, K), device="cuda", generator=g) * 0.05)
    a, ws, qk = dq.dirotq_mxfp4_quantize(x), dq.alloc_mxfp4_workspace(M, K), dq.QkNorm(hq, hk, D)
    gemm_tile(columns)

    def step(y):
        if call == "gemm":
            dq.dirotq_mxfp4_gemm(a, w, y, ws)
        elif call == "linear":
            dq.dirotq_mxfp4_linear(x, w, y, ws)
        else:
            dq.dirotq_mxfp4_qkv(x, w, y, ws, qk)

    want, y = (torch.zeros((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    step(want)
    assert dq.dirotq_workspace_status(ws) == 0
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    run_long(1.3)
    step(y)
    end.record()
    assert dq.dirotq_workspace_status(ws) == 0
    assert start.elapsed_time(end) >= 1290 and torch.equal(y, want)
