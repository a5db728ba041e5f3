"""Norm and rotation of q and k on the GPU, alone, behind a prepared layer, and in the MXFP4 product's epilogue, against 64 bits."""
import pytest
import torch

import mx_reference as ref
from paper_2605_16732_b200 import binding as dq

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Setup:
    def __init__(self, M, hq, hk, D, rot, style, dtype, seed, weights=True, norm=True, positions=True, P=None, w_dtype=None, eps=1e-6):
        g = _gen(seed)
        self.M, self.hq, self.hk, self.D, self.rot, self.style, self.dtype, self.norm, self.eps = M, hq, hk, D, rot, style, dtype, norm, eps
        P = P or M + 9
        self.wq, self.wk = [(1 + 0.3 * torch.randn(D, device="cuda", generator=g)).to(w_dtype or dtype) if weights else None for _ in range(2)]
        angle = torch.arange(P, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / max(rot, 1))
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        self.positions = torch.randint(0, P, (M,), device="cuda", generator=g).to(torch.int32) if positions else None
        self.plan = dq.QkNorm(hq, hk, D, q_weight=self.wq, k_weight=self.wk, eps=eps, norm=norm, rope=style if rot else None, rot_dim=rot, cos=self.cos, sin=self.sin,
                              positions=self.positions)
        self.width = (hq + 2 * hk) * D
        self.x = (torch.randn((M, self.width), device="cuda", generator=g) * torch.exp2(torch.randint(-3, 4, (M, 1), device="cuda", generator=g).float())).to(dtype)

    def want(self, x=None):
        """(q, k, v) and the tolerances of q and k, in 64 bits."""
        x = (self.x if x is None else x).double().view(self.M, -1, self.D)
        at = self.positions.long() if self.positions is not None else torch.arange(self.M, device="cuda")
        out = []
        for part, w in ((x[:, :self.hq], self.wq), (x[:, self.hq:self.hq + self.hk], self.wk)):
            y, mass = ref.head(part, w, self.eps, self.cos[at.clamp(0, len(self.cos) - 1)], self.sin[at.clamp(0, len(self.cos) - 1)], self.style, self.rot, self.norm)
            out.append((y.flatten(1), ref.head_tolerance(y, mass, self.D, self.dtype).flatten(1)))
        return out[0], out[1], x[:, self.hq + self.hk:].flatten(1)


def _within(y, want, tol):
    worst = ((y.double() - want).abs() / tol).max().item()
    assert worst <= 1, worst


CASES = [  # M, q heads, kv heads, head_dim, rotated, style
    (1, 1, 1, 8, 8, "pairs"), (1, 32, 8, 128, 128, "halves"), (3, 5, 5, 64, 64, "pairs"), (7, 16, 16, 72, 36, "halves"), (7, 16, 16, 72, 72, "halves"),
    (33, 14, 2, 128, 64, "pairs"), (5, 3, 1, 256, 256, "halves"), (64, 24, 24, 128, 128, "pairs"), (9, 6, 3, 96, 2, "pairs"), (4, 4, 4, 32, 16, "halves"),
    (11, 7, 1, 40, 0, None), (300, 8, 2, 160, 80, "halves"), (2, 9, 9, 24, 24, "pairs"),
    (6, 4, 2, 8, 4, "halves"), (5, 3, 3, 64, 32, "halves"), (3, 4, 1, 128, 64, "halves"), (4, 2, 2, 128, 48, "halves"), (3, 2, 1, 72, 10, "halves"), (400, 16, 16, 72, 36, "halves"), (2500, 3, 2, 16, 8, "halves"),
    (2600, 5, 1, 128, 128, "pairs")]


@pytest.mark.parametrize("M,hq,hk,D,rot,style", CASES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_norm_and_rotation(M, hq, hk, D, rot, style, dtype):
    s = Setup(M, hq, hk, D, rot, style, DTYPES[dtype], M + D)
    q, k, v = (torch.empty((M, n * D), dtype=s.dtype, device="cuda") for n in (hq, hk, hk))
    before = s.x.clone()
    dq.dirotq_qk_norm_rope(s.x, s.plan, q, k, v)
    (wq, tq), (wk, tk), wv = s.want()
    _within(q, wq, tq)
    _within(k, wk, tk)
    assert torch.equal(v.double(), wv) and torch.equal(s.x, before)
    # in place, v left alone
    y = s.x.clone()
    dq.dirotq_qk_norm_rope(y, s.plan, y[:, :hq * D], y[:, hq * D:(hq + hk) * D])
    assert torch.equal(y[:, :hq * D], q) and torch.equal(y[:, hq * D:(hq + hk) * D], k) and torch.equal(y[:, (hq + hk) * D:], s.x[:, (hq + hk) * D:])


@pytest.mark.parametrize("weights,norm,rot,positions", [(False, True, 64, True), (True, False, 64, True), (True, True, 0, True), (True, True, 64, False), (False, False, 32, False)])
@pytest.mark.parametrize("style", ["pairs", "halves"])
def test_parts_left_out(weights, norm, rot, positions, style):
    s = Setup(21, 6, 2, 64, rot, style, torch.bfloat16, 3, weights=weights, norm=norm, positions=positions, w_dtype=torch.float32, eps=1e-3)
    q, k = torch.empty((21, 384), dtype=s.dtype, device="cuda"), torch.empty((21, 128), dtype=s.dtype, device="cuda")
    dq.dirotq_qk_norm_rope(s.x, s.plan, q, k)
    (wq, tq), (wk, tk), _ = s.want()
    _within(q, wq, tq)
    _within(k, wk, tk)


@pytest.mark.parametrize("style", ["pairs", "halves"])
def test_cache_rows_strides_and_padding(style):
    """k and v by slots into a wider cache; tokens whose position or slot is out of range leave no trace."""
    M, hq, hk, D, rows = 50, 8, 2, 128, 300
    s = Setup(M, hq, hk, D, 128, style, torch.bfloat16, 4)
    g = _gen(9)
    slots = torch.randperm(rows, device="cuda", generator=g)[:M].to(torch.int32)
    slots[3], slots[4], slots[49] = -1, rows, 2 ** 31 - 1
    s.positions[7], s.positions[8], s.positions[9] = -1, len(s.cos), -2 ** 31
    wide = torch.full((M, s.width + 24), 7, dtype=s.dtype, device="cuda")
    wide[:, 8:8 + s.width] = s.x
    x = wide[:, 8:8 + s.width]
    q = torch.full((M, hq * D + 16), 5, dtype=s.dtype, device="cuda")
    cache = torch.full((rows, 2, hk * D + 8), 5, dtype=s.dtype, device="cuda")
    dq.dirotq_qk_norm_rope(x, s.plan, q[:, :hq * D], cache[:, 0, :hk * D], cache[:, 1, :hk * D], slots=slots)
    (wq, tq), (wk, tk), wv = s.want()
    skipped = [3, 4, 7, 8, 9, 49]
    live = torch.tensor([m for m in range(M) if m not in skipped], device="cuda")
    _within(q[live, :hq * D], wq[live], tq[live])
    at = slots[live].long()
    _within(cache[at, 0, :hk * D], wk[live], tk[live])
    assert torch.equal(cache[at, 1, :hk * D].double(), wv[live])
    others = torch.ones(rows, dtype=torch.bool, device="cuda")
    others[at] = False
    assert bool((cache[others] == 5).all()) and bool((cache[:, :, hk * D:] == 5).all()) and bool((q[:, hq * D:] == 5).all()) and bool((q[skipped] == 5).all())
    assert bool((wide[:, :8] == 7).all())


def test_cache_beyond_32_bits():
    """A row of a cache more than 2^32 bytes (and 2^31 elements) from its start."""
    rows, width = 17_000_000, 128
    s = Setup(4, 2, 1, 128, 128, "pairs", torch.bfloat16, 5)
    cache = torch.zeros((rows, width), dtype=s.dtype, device="cuda")
    slots = torch.tensor([rows - 1, 0, rows - 2, 8_500_000], dtype=torch.int32, device="cuda")
    q = torch.empty((4, 256), dtype=s.dtype, device="cuda")
    dq.dirotq_qk_norm_rope(s.x, s.plan, q, cache, slots=slots)
    _, (wk, tk), _ = s.want()
    _within(cache[slots.long()], wk, tk)
    assert int((cache[1:1000] != 0).sum()) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_zeros_infinities_and_nan(dtype):
    s = Setup(6, 2, 2, 64, 64, "halves", DTYPES[dtype], 6, positions=False)
    s.x[1] = 0
    s.x[2, :64], s.x[3, 70], s.x[4, 130] = float("inf"), float("nan"), 0.0
    q, k = torch.empty((6, 128), dtype=s.dtype, device="cuda"), torch.empty((6, 128), dtype=s.dtype, device="cuda")
    dq.dirotq_qk_norm_rope(s.x, s.plan, q, k)
    assert bool((q[1] == 0).all()) and bool((k[1] == 0).all())
    assert bool(torch.isnan(q[2, :64]).all()) and bool(torch.isfinite(q[2, 64:]).all()) and bool(torch.isnan(q[3, 64:]).all()) and bool(torch.isfinite(q[3, :64]).all())
    (wq, tq), (wk, tk), _ = s.want()
    for m in (0, 4, 5):
        _within(q[m], wq[m], tq[m])
        _within(k[m], wk[m], tk[m])


def test_table_rows_of_their_own_stride():
    s = Setup(12, 3, 3, 64, 64, "pairs", torch.bfloat16, 7)
    wide = torch.full((2, len(s.cos), 39), 9.0, device="cuda")
    wide[0, :, :32], wide[1, :, :32] = s.cos, s.sin
    plan = dq.QkNorm(3, 3, 64, q_weight=s.wq, k_weight=s.wk, rope="pairs", cos=wide[0, :, :32], sin=wide[1, :, :32], positions=s.positions)
    outs = [[torch.empty((12, 192), dtype=s.dtype, device="cuda") for _ in range(2)] for _ in range(2)]
    for p, o in zip((s.plan, plan), outs):
        dq.dirotq_qk_norm_rope(s.x, p, *o)
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


# ------------------------------------------------------------------ behind the projections

def _qkv_tolerance(s, proj, mass, K):
    """The epilogue's result against the norm and rotation of the exact projection.  The projection is off by at most d (fp32 sums, as for
    the plain product); with n = h / rms(h), a change d of h changes n by at most (|d_i| + |n_i| rms(d)) / rms(h) to first order (1.01 covers
    the rest at these sizes), a rotation mixes two of those; then the tolerance of the norm and rotation themselves."""
    d = ((-(-K // 64) + 1) * 2.0 ** -22 * mass).view(s.M, -1, s.D)
    h = proj.view(s.M, -1, s.D)
    out = []
    at = s.positions.long() if s.positions is not None else torch.arange(s.M, device="cuda")
    for lo, hi, w in ((0, s.hq, s.wq), (s.hq, s.hq + s.hk, s.wk)):
        hh, dd = h[:, lo:hi], d[:, lo:hi]
        rms = torch.sqrt(hh.square().mean(-1, keepdim=True) + s.eps)
        change = 1.01 * (dd + (hh / rms).abs() * dd.square().mean(-1, keepdim=True).sqrt()) / rms * (1 if w is None else w.double().abs())
        y, m = ref.head(hh, w, s.eps, s.cos[at], s.sin[at], s.style, s.rot, True)
        if s.rot:
            i = torch.arange(s.rot // 2, device="cuda")
            a, b = (2 * i, 2 * i + 1) if s.style == "pairs" else (i, i + s.rot // 2)
            mixed = change.clone()
            mixed[..., a] = mixed[..., b] = change[..., a] + change[..., b]
            change = mixed
        out.append((y.flatten(1), (ref.head_tolerance(y, m, s.D, s.dtype) + change * (1 + torch.finfo(s.dtype).eps)).flatten(1)))
    return out


@pytest.mark.parametrize("M,K,hq,hk,D,style", [(1, 320, 4, 2, 128, "pairs"), (5, 1152, 3, 3, 64, "halves"), (100, 700, 6, 1, 64, "pairs"), (128, 512, 5, 2, 128, "halves"), (130, 512, 5, 2, 128, "pairs"),
                                               (300, 384, 24, 24, 128, "pairs"), (700, 256, 7, 2, 64, "halves"), (257, 640, 2, 1, 64, None)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_mxfp4_qkv(M, K, hq, hk, D, style, dtype):
    s = Setup(M, hq, hk, D, D if style else 0, style, DTYPES[dtype], M + K)
    g = torch.Generator().manual_seed(M)
    x = torch.randn((M, K), generator=g).to(s.dtype)
    w = torch.randn((s.width, K), generator=g) * 0.05
    bias = (torch.randn(s.width, generator=g) * 0.3).to(s.dtype).cuda()
    wq = dq.dirotq_mxfp4_quantize(w.cuda())
    ws = dq.alloc_mxfp4_workspace(M, K)
    y = torch.full((M, s.width + 8), 7, dtype=s.dtype, device="cuda")
    dq.dirotq_mxfp4_qkv(x.cuda(), wq, y[:, :s.width], ws, s.plan, bias=bias)
    assert dq.dirotq_workspace_status(ws) == 0
    proj, mass = ref.product(ref.values(*ref.quantize(x)).cuda(), ref.values(*ref.quantize(w)).cuda(), bias)
    (q, tq), (k, tk) = _qkv_tolerance(s, proj, mass, K)
    nq, nk = hq * D, (hq + hk) * D
    _within(y[:, :nq], q, tq)
    _within(y[:, nq:nk], k, tk)
    _within(y[:, nk:s.width], proj[:, nk:], ref.product_tolerance(proj, mass, K, s.dtype)[:, nk:])
    assert bool((y[:, s.width:] == 7).all())


@pytest.mark.parametrize("M,D,pad", [(3, 64, 5), (140, 64, 3), (9, 128, 1), (150, 128, 7)])
def test_mxfp4_qkv_rows_of_any_alignment(M, D, pad):
    """Rows of y that no wide store can address, and tables with rows of their own: the same bits as aligned ones."""
    s = Setup(M, 3, 2, D, D, "pairs", torch.float16, M)
    g = torch.Generator().manual_seed(5)
    x, w = torch.randn((M, 200), generator=g).half().cuda(), dq.dirotq_mxfp4_quantize((torch.randn((s.width, 200), generator=g) * 0.1).cuda())
    ws = dq.alloc_mxfp4_workspace(M, 200)
    wide = torch.empty((2, len(s.cos), D // 2 + 3), device="cuda")
    wide[0, :, :D // 2], wide[1, :, :D // 2] = s.cos, s.sin
    plan = dq.QkNorm(3, 2, D, q_weight=s.wq, k_weight=s.wk, rope="pairs", cos=wide[0, :, :D // 2], sin=wide[1, :, :D // 2], positions=s.positions)
    y, z = torch.empty((M, s.width), dtype=s.dtype, device="cuda"), torch.full((M, s.width + pad), 7, dtype=s.dtype, device="cuda")
    dq.dirotq_mxfp4_qkv(x, w, y, ws, s.plan)
    dq.dirotq_mxfp4_qkv(x, w, z[:, :s.width], ws, plan)
    assert torch.equal(y, z[:, :s.width]) and bool((z[:, s.width:] == 7).all())


@pytest.mark.parametrize("M", [40, 200])
def test_mxfp4_qkv_padding_tokens(M):
    s = Setup(M, 4, 2, 64, 64, "pairs", torch.bfloat16, 1)
    s.positions[::7] = -1
    s.positions[1::7] = len(s.cos)
    g = torch.Generator().manual_seed(2)
    x, w = torch.randn((M, 256), generator=g).bfloat16().cuda(), dq.dirotq_mxfp4_quantize((torch.randn((s.width, 256), generator=g) * 0.1).cuda())
    ws = dq.alloc_mxfp4_workspace(M, 256)
    y, z = (torch.empty((M, s.width), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dq.dirotq_mxfp4_qkv(x, w, y, ws, s.plan)
    dq.dirotq_mxfp4_linear(x, w, z, ws)
    pad = (s.positions < 0) | (s.positions >= len(s.cos))
    assert torch.equal(y[pad], z[pad]) and torch.equal(y[:, 384:], z[:, 384:]) and not torch.equal(y[~pad], z[~pad])


@pytest.mark.parametrize("M,hq,hk,D,style", [(9, 3, 2, 64, "halves"), (45, 3, 1, 128, "halves"), (150, 3, 1, 64, None), (270, 3, 2, 64, "halves"), (270, 2, 1, 128, "pairs"), (270, 2, 1, 128, "halves")])
@pytest.mark.parametrize("columns", [0, 128, 512])
def test_mxfp4_qkv_alignments_padding_and_plans(M, hq, hk, D, style, columns):
    """One result whatever the alignment of y's rows (none, 16, 32 bytes), the tables' (none, 16, 32 bytes) and the plan; a token out of range keeps its projection."""
    s = Setup(M, hq, hk, D, D if style else 0, style, torch.bfloat16, M + D)
    if style:
        s.positions[::5] = -1
        s.positions[2::7] = len(s.cos)
    g = torch.Generator().manual_seed(3)
    x, w = torch.randn((M, 300), generator=g).bfloat16().cuda(), dq.dirotq_mxfp4_quantize((torch.randn((s.width, 300), generator=g) * 0.1).cuda())
    ws = dq.alloc_mxfp4_workspace(M, 300)
    y, z = (torch.empty((M, s.width), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dq.dirotq_mxfp4_qkv(x, w, y, ws, s.plan)
    dq.dirotq_mxfp4_linear(x, w, z, ws)
    pad = (s.positions < 0) | (s.positions >= len(s.cos)) if style else torch.zeros(M, dtype=torch.bool, device="cuda")
    assert torch.equal(y[pad], z[pad]) and torch.equal(y[:, (hq + hk) * D:], z[:, (hq + hk) * D:]) and not torch.equal(y[~pad], z[~pad])
    try:
        dq.dirotq_set_gemm_tile(columns)
        for more, extra in ((1, 1), (8, 4), (16, 8)):
            wide = torch.full((2, len(s.cos), D // 2 + extra), 9.0, device="cuda")
            wide[0, :, :D // 2], wide[1, :, :D // 2] = (s.cos, s.sin) if style else (0, 0)
            kw = dict(rope=style, cos=wide[0, :, :D // 2], sin=wide[1, :, :D // 2], positions=s.positions) if style else {}
            plan = dq.QkNorm(hq, hk, D, q_weight=s.wq, k_weight=s.wk, eps=s.eps, **kw)
            out = torch.full((M + 1, s.width + more), 7, dtype=torch.bfloat16, device="cuda")
            dq.dirotq_mxfp4_qkv(x, w, out[:M, :s.width], ws, plan)
            assert torch.equal(out[:M, :s.width], y), more
            assert bool((out[M] == 7).all()) and bool((out[:, s.width:] == 7).all())
    finally:
        dq.dirotq_set_gemm_tile(0)
    assert dq.dirotq_workspace_status(ws) == 0


@pytest.mark.parametrize("M,D", [(5, 64), (5, 128), (40, 64), (200, 64), (200, 128)])
def test_mxfp4_qkv_bits_do_not_depend_on_the_plan(M, D):
    s = Setup(M, 4, 1, D, D, "halves", torch.bfloat16, 1)
    g = torch.Generator().manual_seed(2)
    x, w = torch.randn((M, 320), generator=g).bfloat16().cuda(), dq.dirotq_mxfp4_quantize((torch.randn((s.width, 320), generator=g) * 0.1).cuda())
    ws = dq.alloc_mxfp4_workspace(M, 320)
    outs = []
    try:
        for columns in (0, 64, 128, 512):
            dq.dirotq_set_gemm_tile(columns)
            outs.append(torch.empty((M, s.width), dtype=torch.bfloat16, device="cuda"))
            dq.dirotq_mxfp4_qkv(x, w, outs[-1], ws, s.plan)
    finally:
        dq.dirotq_set_gemm_tile(0)
    assert dq.dirotq_workspace_status(ws) == 0
    assert all(torch.equal(o, outs[0]) for o in outs)


def test_mxfp4_qkv_refusals():
    w = dq.dirotq_mxfp4_alloc(768, 64)
    x, y = torch.zeros((8, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((8, 768), dtype=torch.bfloat16, device="cuda")
    ws = dq.alloc_mxfp4_workspace(8, 64)
    cos = torch.zeros((8, 48), device="cuda")
    for plan, status in [(dq.QkNorm(6, 1, 96, rope="pairs", cos=cos, sin=cos), 2), (dq.QkNorm(4, 4, 64, rope="halves", rot_dim=32, cos=cos, sin=cos), 2), (dq.QkNorm(4, 2, 64), 1)]:
        with pytest.raises(dq.DirotqError) as e:
            dq.dirotq_mxfp4_qkv(x, w, y, ws, plan)
        assert e.value.status == status


@pytest.mark.parametrize("fmt", ["int4", "nvfp4", "int4_ph"])
def test_linear_qkv_is_the_layer_and_the_norm(fmt):
    M, K, D, hq, hk = 70, 512, 64, 6, 3
    s = Setup(M, hq, hk, D, D, "pairs", torch.bfloat16, 8)
    g = _gen(3)
    W = 0.05 * torch.randn((K, s.width), device="cuda", generator=g)
    Q, _ = torch.linalg.qr(torch.randn((K, K), dtype=torch.float64, device="cuda", generator=g))
    Q = Q.contiguous()
    layer = dq.dirotq_prepare_layer(W, Q, 32, 64) if fmt == "int4" else dq.dirotq_prepare_layer_nvfp4(W, Q, 32, -8) if fmt == "nvfp4" else \
        dq.dirotq_prepare_layer_ph(W, Q[:, :32].contiguous(), 64)
    x = torch.randn((M, K), device="cuda", generator=g).bfloat16()
    ws = dq.alloc_workspace(layer, M)
    y, z = (torch.empty((M, s.width), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for _ in range(3):
        dq.dirotq_linear_qkv(x, layer, y, ws, s.plan)
    dq.dirotq_linear(x, layer, z, ws)
    q, k = torch.empty((M, hq * D), dtype=torch.bfloat16, device="cuda"), torch.empty((M, hk * D), dtype=torch.bfloat16, device="cuda")
    dq.dirotq_qk_norm_rope(z, s.plan, q, k)
    assert torch.equal(y, torch.cat((q, k, z[:, (hq + hk) * D:]), 1))
    (wq, tq), (wk, tk), _ = s.want(z)
    _within(q, wq, tq)
    _within(k, wk, tk)
    with pytest.raises(dq.DirotqError):
        dq.dirotq_linear_qkv(x, layer, y, ws, dq.QkNorm(6, 2, 64))
    layer.close()


def test_captured_run_of_projection_and_cache_write():
    """The operators as a decoder uses them: project, norm, rotate, write k and v to the cache; captured once, replayed on other tokens."""
    M, K, D, hq, hk, rows = 16, 512, 128, 8, 2, 64
    s = Setup(M, hq, hk, D, D, "halves", torch.bfloat16, 11, P=64)
    g = torch.Generator().manual_seed(4)
    w = dq.dirotq_mxfp4_quantize((torch.randn((s.width, K), generator=g) * 0.05).cuda())
    ws = dq.alloc_mxfp4_workspace(M, K)
    x = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
    slots = torch.empty(M, dtype=torch.int32, device="cuda")
    y, q = torch.empty((M, s.width), dtype=torch.bfloat16, device="cuda"), torch.empty((M, hq * D), dtype=torch.bfloat16, device="cuda")
    cache = torch.zeros((2, rows, hk * D), dtype=torch.bfloat16, device="cuda")

    def step():
        dq.dirotq_mxfp4_linear(x, w, y, ws)
        dq.dirotq_qk_norm_rope(y, s.plan, q, cache[0], cache[1], slots=slots)

    def inputs(i):
        gi = _gen(100 + i)
        return torch.randn((M, K), device="cuda", generator=gi).bfloat16(), torch.randperm(rows, device="cuda", generator=gi)[:M].to(torch.int32), \
            torch.randint(0, 64, (M,), device="cuda", generator=gi).to(torch.int32)

    def load(i):
        for to, value in zip((x, slots, s.positions), inputs(i)):
            to.copy_(value)

    load(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    expect = torch.zeros_like(cache)
    cache.zero_()
    for i in (1, 2, 3):
        load(i)
        graph.replay()
        got = (q.clone(), cache.clone())
        cache.copy_(expect)
        step()
        assert torch.equal(got[0], q) and torch.equal(got[1], cache)
        expect.copy_(cache)
