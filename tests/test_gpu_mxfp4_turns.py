"""The MXFP4 products where every block (or pair of blocks) has several tiles: what is carried from one tile to the next - ring, accumulators and their
hand-back, bias buffers, sums of squares, weights asked for early - in every plan, against 64 bits and one another.  Ragged rows and columns; one, an odd
and an even number of stages a tile, fewer and more of them than the ring holds."""
import pytest
import torch

import mx_reference as ref
from paper_2605_16732_b200 import binding as dq
from test_gpu_qk_norm import Setup, _qkv_tolerance, _within

pytestmark = pytest.mark.gpu
M = 1300  # 6 row blocks of 256, 11 of 128


@pytest.fixture
def gemm_tile():
    yield dq.dirotq_set_gemm_tile
    dq.dirotq_set_gemm_tile(0)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _turns(N, rows, columns, units):
    return -(-(-(-M // rows) * -(-N // columns)) // units)


@pytest.mark.parametrize("K", [96, 700, 1664, 1800])  # 1, 3, 7 and 8 blocks of 256
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_products(K, dtype, gemm_tile):
    N, pad = 9216 + 70, 2
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert _turns(N, 256, 256, sms // 2) >= 3 and _turns(N, 128, 128, sms) >= 3 and _turns(N, 128, 64, sms) >= 3
    g = _gen(K)
    x, w = torch.randn((M, K), generator=g).to(dtype), torch.randn((N, K), generator=g) * 0.05
    bias = torch.randn(N, generator=g).to(dtype).cuda()
    xd, a, b = x.cuda(), dq.dirotq_mxfp4_quantize(x.cuda()), dq.dirotq_mxfp4_quantize(w.cuda())
    want, mass = ref.product(ref.values(*ref.quantize(x)).cuda(), ref.values(*ref.quantize(w)).cuda(), bias)
    tol = ref.product_tolerance(want, mass, K, dtype)
    ws = dq.alloc_mxfp4_workspace(M, K)
    first = None
    for columns in (512, 128, 64, 0):
        gemm_tile(columns)
        for call in range(4):
            y = torch.full((M + 1, N + pad), 7, dtype=dtype, device="cuda")
            if call % 2:
                dq.dirotq_mxfp4_linear(xd, b, y[:M, :N], ws, bias=bias)
            else:
                dq.dirotq_mxfp4_gemm(a, b, y[:M, :N], ws, bias=bias)
            if first is None:
                first = y
                worst = ((y[:M, :N].double() - want).abs() / tol).max().item()
                assert worst <= 1, worst
                assert bool((y[M] == 7).all()) and bool((y[:, N:] == 7).all())
            assert torch.equal(y, first), (columns, call)
    assert dq.dirotq_workspace_status(ws) == 0


@pytest.mark.parametrize("hq,hk,D", [(24, 24, 128), (97, 24, 64), (63, 5, 128)])
@pytest.mark.parametrize("style", ["pairs", "halves", None])
@pytest.mark.parametrize("K", [96, 700, 1800])
def test_fused_qkv(hq, hk, D, style, K, gemm_tile):
    s = Setup(M, hq, hk, D, D if style else 0, style, torch.bfloat16, K + D)
    g = _gen(K)
    x, w = torch.randn((M, K), generator=g).bfloat16(), torch.randn((s.width, K), generator=g) * 0.05
    bias = (torch.randn(s.width, generator=g) * 0.3).bfloat16().cuda()
    xd, b, ws = x.cuda(), dq.dirotq_mxfp4_quantize(w.cuda()), dq.alloc_mxfp4_workspace(M, K)
    proj, mass = ref.product(ref.values(*ref.quantize(x)).cuda(), ref.values(*ref.quantize(w)).cuda(), bias)
    (q, tq), (k, tk) = _qkv_tolerance(s, proj, mass, K)
    nq, nk = hq * D, (hq + hk) * D
    first = None
    for columns in (512, 128, 64, 0) if D == 64 else (512, 128, 0):
        gemm_tile(columns)
        for call in range(2):
            y = torch.full((M + 1, s.width + 8), 7, dtype=torch.bfloat16, device="cuda")
            dq.dirotq_mxfp4_qkv(xd, b, y[:M, :s.width], ws, s.plan, bias=bias)
            if first is None:
                first = y
                _within(y[:M, :nq], q, tq)
                _within(y[:M, nq:nk], k, tk)
                _within(y[:M, nk:s.width], proj[:, nk:], ref.product_tolerance(proj, mass, K, torch.bfloat16)[:, nk:])
                assert bool((y[M] == 7).all()) and bool((y[:, s.width:] == 7).all())
            assert torch.equal(y, first), (columns, call)
    assert dq.dirotq_workspace_status(ws) == 0


@pytest.mark.parametrize("columns", [512, 128, 0])
def test_consecutive_layers(columns, gemm_tile):
    """Layers one behind the other on one stream, each from the one before it, with weights of their own: no stage keeps what an earlier call left."""
    K = N = 1536  # (few column blocks: 36 pair tiles; the chain below is what is tested)
    g = _gen(7)
    ws = dq.alloc_mxfp4_workspace(4000, K)
    weights = [dq.dirotq_mxfp4_quantize((torch.randn((N, K), generator=g) * 0.04).cuda()) for _ in range(3)]
    x = torch.randn((4000, K), generator=g).bfloat16().cuda()
    gemm_tile(columns)
    apart = [x]
    for w in weights:
        torch.cuda.synchronize()
        apart.append(torch.empty_like(x))
        dq.dirotq_mxfp4_linear(apart[-2], w, apart[-1], ws)
    torch.cuda.synchronize()
    for _ in range(5):
        outs = [x] + [torch.zeros_like(x) for _ in weights]
        for i, w in enumerate(weights):
            dq.dirotq_mxfp4_linear(outs[i], w, outs[i + 1], ws)
        assert all(torch.equal(a, b) for a, b in zip(outs, apart))
    assert dq.dirotq_workspace_status(ws) == 0
