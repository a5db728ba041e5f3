"""MXFP4 on the GPU: quantizer, plain import and export, products, against the definitions in 64 bits."""
import pytest
import torch

import mx_reference as ref
from paper_2605_16732_b200 import binding as dq

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _data(rows, K, seed, dtype=torch.float32):
    g = _gen(seed)
    x = torch.randn((rows, K), generator=g) * torch.exp2(torch.randint(-6, 7, (rows, 1), generator=g).float())
    x[:, torch.randint(0, K, (max(1, K // 64),), generator=g)] *= 40
    return x.to(dtype)


def _strided(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + pad), 7, dtype=t.dtype, device="cuda")
    view = wide[:, :t.shape[1]]
    view.copy_(t)
    return view


def _numbers(t):
    """NaN as a number, so that tensors can be compared."""
    return torch.where(torch.isnan(t), 123.456, t)


def _check_quantized(t, x, rule):
    codes, scales = ref.quantize(x, rule)
    got_codes, got_scales = dq.dirotq_mxfp4_export(t)
    assert torch.equal(got_scales.cpu(), scales)
    assert torch.equal(ref.unpack(got_codes.cpu(), x.shape[1]), codes)
    return codes, scales


@pytest.mark.parametrize("rows,K,pad", [(1, 1, 0), (1, 31, 0), (1, 32, 0), (3, 33, 0), (5, 64, 3), (130, 257, 0), (257, 256, 8), (64, 1152, 0), (300, 4600, 5), (2, 40000, 16)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rule", [ref.FLOOR, ref.CEIL])
def test_quantize_rows_and_back(rows, K, pad, dtype, rule):
    x = _data(rows, K, rows * 7 + K, DTYPES[dtype])
    t = dq.dirotq_mxfp4_quantize(_strided(x, pad), scale_rule=rule)
    codes, scales = _check_quantized(t, x, rule)
    want = ref.values(codes, scales)
    for out_dtype in DTYPES.values():
        y = torch.full((rows, K + pad), 7, dtype=out_dtype, device="cuda")
        dq.dirotq_mxfp4_dequantize(t, y[:, :K])
        assert torch.equal(y[:, :K].cpu(), want.to(out_dtype))
        assert bool((y[:, K:] == 7).all())


@pytest.mark.parametrize("rows,K,pad", [(1, 1, 0), (31, 33, 0), (33, 256, 0), (257, 300, 7), (1152, 640, 0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_quantize_columns(rows, K, pad, dtype):
    x = _data(rows, K, rows + K, DTYPES[dtype])
    for rule in (ref.FLOOR, ref.CEIL):
        t = dq.dirotq_mxfp4_quantize(_strided(x.T.contiguous(), pad), scale_rule=rule, layout=dq.LAYOUT_KN)
        _check_quantized(t, x, rule)


@pytest.mark.parametrize("layout", [dq.LAYOUT_NK, dq.LAYOUT_KN])
def test_quantize_special_values(layout):
    """A row per case: zeros, ties, saturation, an infinity or a NaN in one block, subnormal numbers, the largest ones, negative zeros."""
    inf, nan = float("inf"), float("nan")
    tiny, big = 2.0 ** -149, torch.finfo(torch.float32).max
    x = torch.zeros((12, 96))
    x[1, :16] = torch.tensor([4.0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5.0, 7.9])
    x[2, 32:36] = torch.tensor([7.99, -7.99, 6.01, 5.0])
    x[3, 40], x[3, 0], x[3, 95] = inf, 1.0, -2.0
    x[4, 5], x[4, 50], x[4, 6] = nan, 3.0, inf
    x[5, 10] = -inf
    x[6, 0], x[6, 33], x[6, 64], x[6, 65] = tiny, 2.0 ** -126, 3 * tiny, 2.0 ** -130
    x[7, 0], x[7, 1], x[7, 32], x[7, 64] = big, -big / 3, 2.0 ** 127, 1.6 * 2.0 ** 127
    x[8, :] = -0.0
    x[9, 0], x[9, 1], x[9, 2] = 1.0, -1e-30, 2.0 ** -100
    x[10, :3] = torch.tensor([2.0 ** -125, 2.0 ** -128, -(2.0 ** -126)])
    x[11, :] = torch.linspace(-6, 6, 96)
    for rule in (ref.FLOOR, ref.CEIL):
        d = x.cuda() if layout == dq.LAYOUT_NK else x.T.contiguous().cuda()
        t = dq.dirotq_mxfp4_quantize(d, scale_rule=rule, layout=layout)
        codes, scales = _check_quantized(t, x, rule)
        y = torch.empty((12, 96), device="cuda")
        dq.dirotq_mxfp4_dequantize(t, y)
        # (values are compared as the fp32 numbers they round to: 4 * 2^126, from the largest numbers, is an infinity there)
        assert torch.equal(_numbers(y.cpu()), _numbers(ref.values(codes, scales).float()))
        assert bool(torch.isnan(y[3, 32:64]).all()) and bool(torch.isfinite(y[3, :32]).all()) and bool(torch.isfinite(y[3, 64:]).all())
        if rule == ref.CEIL:
            finite = torch.isfinite(x).all(1) & torch.isfinite(y.cpu()).all(1)
            assert bool(((y.cpu() - x).abs()[finite] <= x.abs().unflatten(1, (3, 32)).amax(2, keepdim=True).expand(-1, -1, 32).flatten(1)[finite]).all())


@pytest.mark.parametrize("rows,K", [(1, 1), (3, 31), (130, 33), (257, 513), (64, 4096)])
def test_import_and_export(rows, K):
    g = _gen(rows + K)
    packed = torch.randint(0, 256, (rows, -(-K // 2)), generator=g, dtype=torch.uint8)
    scales = torch.randint(0, 256, (rows, -(-K // 32)), generator=g, dtype=torch.uint8)
    t = dq.dirotq_mxfp4_import(packed.cuda(), scales.cuda(), K)
    got, got_scales = dq.dirotq_mxfp4_export(t)
    if K % 2:
        packed[:, -1] &= 15
    assert torch.equal(got.cpu(), packed) and torch.equal(got_scales.cpu(), scales)
    y = torch.empty((rows, K), device="cuda")
    dq.dirotq_mxfp4_dequantize(t, y)
    want = ref.values(ref.unpack(packed, K), scales).float()
    assert torch.equal(_numbers(y.cpu()), _numbers(want))


def _operand(rows, K, seed, spread=6):
    """Random codes, scales of a spread of powers of two: (operand, values in 64 bits on the GPU)."""
    g = _gen(seed)
    codes = torch.randint(0, 16, (rows, K), generator=g, dtype=torch.uint8)
    scales = torch.randint(127 - spread, 128 + spread, (rows, -(-K // 32)), generator=g, dtype=torch.uint8)
    t = dq.dirotq_mxfp4_import(ref.pack(codes).cuda(), scales.cuda(), K)
    return t, ref.values(codes.cuda(), scales.cuda())


def _close(y, want, mass, K):
    tol = ref.product_tolerance(want, mass, K, y.dtype)
    top = torch.finfo(y.dtype).max
    over = want.abs() - tol > top  # rounds to an infinity
    assert torch.equal(y[over].double(), torch.sign(want[over]) * float("inf"))
    near = (want.abs() + tol > top) & ~over & torch.isinf(y)  # may
    want, y = torch.where(over | near, 0.0, want), torch.where(over | near, 0.0, y)
    worst = ((y.double() - want).abs() / tol).max().item()
    assert worst <= 1, worst


SIZES = [(1, 1, 1), (1, 130, 32), (2, 64, 64), (7, 33, 65), (16, 1152, 1152), (33, 200, 2050), (64, 72, 12288), (127, 129, 257), (128, 128, 256), (129, 257, 300), (255, 300, 4600), (300, 130, 96),
         (512, 1157, 1152), (1000, 2304, 700), (2500, 1500, 640)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("with_bias,pad", [(True, 0), (False, 5), (True, 8)])
def test_gemm(M, N, K, dtype, with_bias, pad):
    a, av = _operand(M, K, M + K, 3)
    b, bv = _operand(N, K, 3 * N + K, 3)
    dt = DTYPES[dtype]
    bias = (torch.randn(N, generator=_gen(N)) * 3).to(dt).cuda() if with_bias else None
    want, mass = ref.product(av, bv, bias)
    if dt is torch.float16 and want.abs().max() > 60000:
        pytest.skip("beyond fp16")
    y = torch.full((M, N + pad), 7, dtype=dt, device="cuda")
    ws = dq.alloc_mxfp4_workspace(M, K)
    dq.dirotq_mxfp4_gemm(a, b, y[:, :N], ws, bias=bias)
    assert dq.dirotq_workspace_status(ws) == 0
    _close(y[:, :N], want, mass, K)
    assert bool((y[:, N:] == 7).all())


def test_gemm_scales_over_their_range():
    """Scales from 2^-60 to 2^60 on one side and their counterparts on the other: every byte value is applied as that power of two."""
    K, M, N = 1024, 130, 140
    g = _gen(5)
    s = torch.randint(-60, 61, (1, K // 32), generator=g)
    ca, cb = (torch.randint(0, 16, (n, K), generator=g, dtype=torch.uint8) for n in (M, N))
    sa, sb = (127 + s).to(torch.uint8).expand(M, -1).contiguous(), (127 - s).to(torch.uint8).expand(N, -1).contiguous()
    a, b = (dq.dirotq_mxfp4_import(ref.pack(c).cuda(), t.cuda(), K) for c, t in ((ca, sa), (cb, sb)))
    want, mass = ref.product(ref.values(ca, sa).cuda(), ref.values(cb, sb).cuda())
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    dq.dirotq_mxfp4_gemm(a, b, y, dq.alloc_mxfp4_workspace(M, K))
    _close(y, want, mass, K)


@pytest.mark.parametrize("M", [3, 200])
def test_nan_blocks_reach_their_rows_and_columns_only(M):
    K, N = 200, 150
    a, av = _operand(M, K, 1, 2)
    b, bv = _operand(N, K, 2, 2)
    ca, sa = dq.dirotq_mxfp4_export(a)
    cb, sb = dq.dirotq_mxfp4_export(b)
    sa[2, 3] = 255
    sb[140, 6] = 255  # the ragged last block
    a, b = dq.dirotq_mxfp4_import(ca, sa, K, out=a), dq.dirotq_mxfp4_import(cb, sb, K, out=b)
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    dq.dirotq_mxfp4_gemm(a, b, y, dq.alloc_mxfp4_workspace(M, K))
    nan = torch.isnan(y)
    want = torch.zeros_like(nan)
    want[2], want[:, 140] = True, True
    assert torch.equal(nan, want)
    clean, mass = ref.product(av, bv)
    keep = ~want
    assert bool(((y.double() - clean).abs() <= ref.product_tolerance(clean, mass, K, y.dtype))[keep].all())


def test_scale_padding_is_written_over_old_contents():
    """A buffer that held NaN scales in the place of what is now padding behind K."""
    M, N, K = 40, 30, 70
    buffers = []
    for rows in (M, N):
        t = dq.dirotq_mxfp4_alloc(rows, K)
        t.buffer.fill_(255)
        buffers.append(t)
    x, w = _data(M, K, 1), _data(N, K, 2)
    a = dq.dirotq_mxfp4_quantize(x.cuda(), out=buffers[0])
    b = dq.dirotq_mxfp4_quantize(w.T.contiguous().cuda(), out=buffers[1], layout=dq.LAYOUT_KN)
    want, mass = ref.product(*(ref.values(*ref.quantize(t)).cuda() for t in (x, w)))
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    dq.dirotq_mxfp4_gemm(a, b, y, dq.alloc_mxfp4_workspace(M, K))
    _close(y, want, mass, K)


@pytest.mark.parametrize("N,K", [(9216, 1152), (1157, 700), (300, 4608)])
def test_a_rows_bits_do_not_depend_on_the_other_rows(N, K):
    x = _data(700, K, 3, torch.bfloat16).cuda()
    w = dq.dirotq_mxfp4_quantize(_data(N, K, 4).cuda())
    ws = dq.alloc_mxfp4_workspace(700, K)
    y = torch.empty((700, N), dtype=torch.bfloat16, device="cuda")
    dq.dirotq_mxfp4_linear(x, w, y, ws)
    for M in (1, 2, 8, 17, 64, 65, 128, 129, 256, 400, 699):
        z = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
        dq.dirotq_mxfp4_linear(x[:M], w, z, ws)
        assert torch.equal(z, y[:M]), M
    assert dq.dirotq_workspace_status(ws) == 0


@pytest.mark.parametrize("M,N,K,pad", [(1, 300, 1152, 0), (5, 64, 33, 3), (130, 257, 512, 16), (1500, 768, 700, 0)])
@pytest.mark.parametrize("x_dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rule", [ref.FLOOR, ref.CEIL])
def test_linear(M, N, K, pad, x_dtype, rule):
    x, w = _data(M, K, M, DTYPES[x_dtype]), _data(N, K, N) * 0.02
    wq = dq.dirotq_mxfp4_quantize(w.cuda(), scale_rule=rule)
    bias = torch.randn(N, generator=_gen(1)).bfloat16().cuda()
    ws = dq.alloc_mxfp4_workspace(M + 3, K)
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    dq.dirotq_mxfp4_linear(_strided(x, pad), wq, y, ws, bias=bias, scale_rule=rule)
    want, mass = ref.product(ref.values(*ref.quantize(x, rule)).cuda(), ref.values(*ref.quantize(w, rule)).cuda(), bias)
    _close(y, want, mass, K)
    z = torch.empty_like(y)
    dq.dirotq_mxfp4_gemm(dq.dirotq_mxfp4_quantize(x.cuda(), scale_rule=rule), wq, z, ws, bias=bias)
    assert torch.equal(y, z)


@pytest.fixture
def gemm_tile():
    yield dq.dirotq_set_gemm_tile
    dq.dirotq_set_gemm_tile(0)


@pytest.mark.parametrize("M,N,K,pad", [(1, 65, 40, 0), (9, 200, 700, 3), (16, 1157, 1152, 0), (130, 64, 4600, 0), (300, 1157, 512, 11), (257, 2304, 1152, 0), (2000, 320, 300, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_every_plan_gives_the_same_bits(M, N, K, pad, dtype, gemm_tile):
    x = (_data(M, K, 3) * 0.1).to(DTYPES[dtype])
    w = dq.dirotq_mxfp4_quantize(_data(N, K, 4).cuda())
    bias = torch.randn(N, generator=_gen(2)).to(DTYPES[dtype]).cuda()
    ws = dq.alloc_mxfp4_workspace(M, K)
    a = dq.dirotq_mxfp4_quantize(x.cuda())
    want, mass = ref.product(ref.values(*ref.quantize(x)).cuda(), ref.values(*ref.quantize(_data(N, K, 4))).cuda(), bias)
    first = None
    for columns in (0, 64, 128, 512):
        gemm_tile(columns)
        for fused in (False, True):
            y = torch.full((M, N + pad), 7, dtype=DTYPES[dtype], device="cuda")
            if fused:
                dq.dirotq_mxfp4_linear(x.cuda(), w, y[:, :N], ws, bias=bias)
            else:
                dq.dirotq_mxfp4_gemm(a, w, y[:, :N], ws, bias=bias)
            assert dq.dirotq_workspace_status(ws) == 0
            if first is None:
                first = y.clone()
                _close(y[:, :N], want, mass, K)
            assert torch.equal(y, first), (columns, fused)


def test_captured_graph_another_stream_and_two_workspaces():
    M, N, K = 200, 384, 512
    w = dq.dirotq_mxfp4_quantize(_data(N, K, 1).cuda())
    xs = [_data(M, K, 10 + i, torch.bfloat16).cuda() for i in range(3)]
    want = []
    for x in xs:
        y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
        dq.dirotq_mxfp4_linear(x, w, y, dq.alloc_mxfp4_workspace(M, K))
        want.append(y)
    torch.cuda.synchronize()
    # two calls at once on two streams, each with a workspace of its own
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [dq.alloc_mxfp4_workspace(M, K) for _ in range(2)]
    outs = [torch.empty_like(want[0]) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            dq.dirotq_mxfp4_linear(xs[i], w, outs[i], spaces[i], stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, t) for o, t in zip(outs, want))
    # captured, replayed on new inputs
    x, y = xs[0].clone(), torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        dq.dirotq_mxfp4_linear(x, w, y, spaces[0])
    for i in (2, 1, 0):
        x.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i])
    assert dq.dirotq_workspace_status(spaces[0]) == 0


def test_operands_made_on_another_stream():
    """Memory that the current stream is still to write is handed out again: an operand made in it on another stream comes after."""
    rows, K = 300, 4096
    x = _data(rows, K, 1, torch.bfloat16).cuda()
    codes, scales = ref.quantize(x.cpu())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for make in (lambda: dq.dirotq_mxfp4_quantize(x, stream=side), lambda: dq.dirotq_mxfp4_import(ref.pack(codes).cuda(), scales.cuda(), K, stream=side)):
        old = dq.dirotq_mxfp4_alloc(rows, K)
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        old.buffer.fill_(255)
        where = old.buffer.data_ptr()
        old.close()
        del old
        t = make()
        torch.cuda.synchronize()
        got, got_scales = dq.dirotq_mxfp4_export(t)
        assert torch.equal(ref.unpack(got.cpu(), K), codes) and torch.equal(got_scales.cpu(), scales), where == t.buffer.data_ptr()


@pytest.mark.parametrize("M", [4, 40, 300])
def test_weights_quantized_right_before_the_call(M):
    """The product's weights come from the kernel just before the activations' quantizer: nothing of them is read too early."""
    N, K = 4096, 2048
    ws = dq.alloc_mxfp4_workspace(M, K)
    x = _data(M, K, 1, torch.bfloat16).cuda()
    w = dq.dirotq_mxfp4_alloc(N, K)
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    weights = [_data(N, K, 20 + i).cuda() for i in range(2)]
    want = []
    for v in weights:
        dq.dirotq_mxfp4_quantize(v, out=w)
        torch.cuda.synchronize()
        dq.dirotq_mxfp4_linear(x, w, y, ws)
        want.append(y.clone())
        torch.cuda.synchronize()
    for i in range(20):
        dq.dirotq_mxfp4_quantize(weights[i & 1], out=w)
        dq.dirotq_mxfp4_linear(x, w, y, ws)
        assert torch.equal(y, want[i & 1]), i


@pytest.mark.parametrize("layout", [dq.LAYOUT_NK, dq.LAYOUT_KN])
def test_rows_beyond_32_bits(layout):
    """Rows so far apart that the last one starts more than 2^31 elements (2^32 bytes) behind the first."""
    apart, n, w = 2 ** 27 + 16, 20, 64
    x = torch.empty(19 * apart + w, dtype=torch.bfloat16, device="cuda").as_strided((n, w), (apart, 1))
    data = _data(n, w, 1, torch.bfloat16)
    x.copy_(data)
    t = dq.dirotq_mxfp4_quantize(x, layout=layout)
    as_rows = data if layout == dq.LAYOUT_NK else data.T.contiguous()
    codes, scales = _check_quantized(t, as_rows, ref.FLOOR)
    if layout == dq.LAYOUT_NK:
        dq.dirotq_mxfp4_dequantize(t, x)
        assert torch.equal(x.cpu(), ref.values(codes, scales).to(torch.bfloat16))
        b, bv = _operand(48, w, 5, 3)
        want, mass = ref.product(ref.values(codes, scales).cuda(), bv)
        dq.dirotq_mxfp4_gemm(t, b, x[:, :48], dq.alloc_mxfp4_workspace(n, w))
        _close(x[:, :48], want, mass, w)


@pytest.mark.parametrize("M", [2, 60])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_linear_of_infinities_and_nan(M, dtype):
    """A NaN block of the activations reaches its own row only, whichever kernel quantizes it."""
    K, N = 300, 70
    x = _data(M, K, 1, DTYPES[dtype])
    x[1, 299] = float("inf")
    x[0, 5] = float("-inf") if M > 2 else x[0, 5]
    w = dq.dirotq_mxfp4_quantize(_data(N, K, 2).cuda())
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    dq.dirotq_mxfp4_linear(x.cuda(), w, y, dq.alloc_mxfp4_workspace(M, K))
    bad = ~torch.isfinite(x).all(1).cuda()
    assert bool(torch.isnan(y[bad]).all()) and bool(torch.isfinite(y[~bad]).all())


def test_an_operand_times_itself_and_a_reused_handle():
    K = 300
    a, av = _operand(200, K, 1, 2)
    ws = dq.alloc_mxfp4_workspace(200, K)
    y = torch.empty((200, 200), dtype=torch.bfloat16, device="cuda")
    dq.dirotq_mxfp4_gemm(a, a, y, ws)
    want, mass = ref.product(av, av)
    _close(y, want, mass, K)
    x = _data(200, K, 9)
    dq.dirotq_mxfp4_quantize(x.cuda(), out=a)
    v = ref.values(*ref.quantize(x)).cuda()
    dq.dirotq_mxfp4_gemm(a, a, y, ws)
    want, mass = ref.product(v, v)
    _close(y, want, mass, K)


def test_refusals_with_handles():
    a, b = dq.dirotq_mxfp4_alloc(8, 64), dq.dirotq_mxfp4_alloc(16, 96)
    c = dq.dirotq_mxfp4_alloc(16, 64)
    L = dq.lib()
    y = torch.empty((8, 16), dtype=torch.bfloat16, device="cuda")
    ws = dq.alloc_mxfp4_workspace(8, 64)
    gemm = lambda a, b, y_ptr=y.data_ptr(), dt=1, ldy=16, w=ws.data_ptr(), n=ws.numel(): L.dirotq_mxfp4_gemm(a.handle, b.handle, None, y_ptr, dt, ldy, w, n, None)
    assert gemm(a, b) == 1                                    # other K
    assert gemm(a, c, dt=0) == 1 and gemm(a, c, ldy=15) == 1  # fp32 output, short rows
    assert gemm(a, c, y_ptr=y.data_ptr() + 1) == 1 and gemm(a, c, y_ptr=None) == 1
    assert gemm(a, c, w=None) == 1 and gemm(a, c, w=ws.data_ptr() + 8) == 1 and gemm(a, c, n=128) == 3
    x = torch.zeros((8, 64), dtype=torch.bfloat16, device="cuda")
    lin = lambda x_ptr=x.data_ptr(), dt=1, ldx=64, M=8, rule=0, w=ws.data_ptr(), n=ws.numel(): L.dirotq_mxfp4_linear(
        x_ptr, dt, ldx, M, rule, c.handle, None, y.data_ptr(), 1, 16, w, n, None)
    assert lin(dt=2) == 1 and lin(ldx=63) == 1 and lin(M=0) == 1 and lin(rule=2) == 1 and lin(x_ptr=x.data_ptr() + 1) == 1 and lin(x_ptr=None) == 1
    assert lin(w=ws.data_ptr() + 16) == 1 and lin(n=1024) == 3
    q = lambda x_ptr=x.data_ptr(), dt=1, layout=1, ld=64, rule=0: L.dirotq_mxfp4_quantize(x_ptr, dt, layout, ld, rule, a.handle, None)
    assert q(dt=2) == 1 and q(layout=2) == 1 and q(ld=63) == 1 and q(layout=0, ld=7) == 1 and q(rule=-1) == 1 and q(x_ptr=None) == 1
    assert L.dirotq_mxfp4_dequantize(a.handle, x.data_ptr(), 1, 63, None) == 1
    a.close()
    with pytest.raises(Exception):
        dq.dirotq_mxfp4_gemm(a, c, y, ws)
