"""Forms of the calls on a fused q/k/v weight: without norm, without weights, x in 32 bits, the other scale rule, infinities and NaN, through the product's
epilogue with the activations quantized by its own blocks (few tokens) and before it (many); and behind prepared layers of every format."""
import pytest
import torch

import mx_reference as ref
from paper_2605_16732_b200 import binding as dq
from test_gpu_qk_norm import Setup, _gen, _qkv_tolerance, _within

pytestmark = pytest.mark.gpu


def _rotated_only(s, proj, mass, K):
    """Norm left out: the projection's own error (as in the plain product's tolerance, without its rounding) through the rotation, which mixes two of them,
    then the rotation's two products and addition, and the one rounding."""
    d = ((-(-K // 64) + 1) * 2.0 ** -22 * mass).view(s.M, -1, s.D)
    h = proj.view(s.M, -1, s.D)
    at = s.positions.long()
    out = []
    for lo, hi in ((0, s.hq), (s.hq, s.hq + s.hk)):
        y, m = ref.head(h[:, lo:hi], None, s.eps, s.cos[at], s.sin[at], s.style, s.rot, False)
        change = d[:, lo:hi]
        if s.rot:
            i = torch.arange(s.rot // 2, device="cuda")
            a, b = (2 * i, 2 * i + 1) if s.style == "pairs" else (i, i + s.rot // 2)
            mixed = change.clone()
            mixed[..., a] = mixed[..., b] = change[..., a] + change[..., b]
            change = mixed
        out.append((y.flatten(1), (ref.head_tolerance(y, m, s.D, s.dtype) + change * (1 + torch.finfo(s.dtype).eps)).flatten(1)))
    return out


@pytest.mark.parametrize("M", [3, 70, 300])  # (3 tokens of 700 elements: quantized by the product's own blocks)
@pytest.mark.parametrize("D,style", [(64, "pairs"), (64, "halves"), (128, "pairs"), (128, "halves"), (128, None)])
@pytest.mark.parametrize("norm,weights", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("x_dtype,rule", [(torch.float32, dq.MX_SCALE_FLOOR), (torch.bfloat16, dq.MX_SCALE_CEIL)])
def test_parts_left_out(M, D, style, norm, weights, x_dtype, rule):
    K, hq, hk = 700, 5, 2
    s = Setup(M, hq, hk, D, D if style else 0, style, torch.bfloat16, M + D, weights=weights, norm=norm, eps=1e-3)
    g = torch.Generator().manual_seed(M)
    x, w = torch.randn((M, K), generator=g).to(x_dtype), torch.randn((s.width, K), generator=g) * 0.05
    bias = (torch.randn(s.width, generator=g) * 0.3).bfloat16().cuda()
    b, ws = dq.dirotq_mxfp4_quantize(w.cuda(), scale_rule=rule), dq.alloc_mxfp4_workspace(M, K)
    y = torch.empty((M, s.width), dtype=torch.bfloat16, device="cuda")
    dq.dirotq_mxfp4_qkv(x.cuda(), b, y, ws, s.plan, bias=bias, scale_rule=rule)
    assert dq.dirotq_workspace_status(ws) == 0
    proj, mass = ref.product(ref.values(*ref.quantize(x, rule)).cuda(), ref.values(*ref.quantize(w, rule)).cuda(), bias)
    if not norm:
        s.wq = s.wk = None
    (q, tq), (k, tk) = (_qkv_tolerance if norm else _rotated_only)(s, proj, mass, K)
    nq, nk = hq * D, (hq + hk) * D
    _within(y[:, :nq], q, tq)
    _within(y[:, nq:nk], k, tk)
    _within(y[:, nk:], proj[:, nk:], ref.product_tolerance(proj, mass, K, torch.bfloat16)[:, nk:])


@pytest.mark.parametrize("M", [3, 300])
@pytest.mark.parametrize("D,style", [(64, "pairs"), (64, "halves"), (128, "pairs"), (128, "halves")])
def test_infinities_and_nan(M, D, style):
    """A token with an infinity or a NaN is NaN throughout and changes no other; a weight row with a NaN block makes its head NaN in q and k, its column alone
    in v, and nothing else."""
    K, hq, hk = 320, 3, 2
    s = Setup(M, hq, hk, D, D, style, torch.bfloat16, M)
    g = torch.Generator().manual_seed(5)
    x, w = torch.randn((M, K), generator=g).bfloat16().cuda(), (torch.randn((s.width, K), generator=g) * 0.05).cuda()
    ws = dq.alloc_mxfp4_workspace(M, K)

    def run(x, w):
        y = torch.empty((M, s.width), dtype=torch.bfloat16, device="cuda")
        dq.dirotq_mxfp4_qkv(x, dq.dirotq_mxfp4_quantize(w), y, ws, s.plan)
        return y

    clean = run(x, w)
    assert bool(torch.isfinite(clean).all())
    bad = x.clone()
    bad[0, 319], bad[2, 7] = float("-inf"), float("nan")
    y = run(bad, w)
    rows = torch.zeros(M, dtype=torch.bool, device="cuda")
    rows[0] = rows[2] = True
    assert bool(torch.isnan(y[rows]).all()) and torch.equal(y[~rows], clean[~rows])
    bad = w.clone()
    bad[D + 5, 100], bad[(hq + hk) * D + 9, 0] = float("inf"), float("nan")
    y = run(x, bad)
    cols = torch.zeros(s.width, dtype=torch.bool, device="cuda")
    cols[D:2 * D] = cols[(hq + hk) * D + 9] = True
    assert bool(torch.isnan(y[:, cols]).all()) and torch.equal(y[:, ~cols], clean[:, ~cols])
    assert dq.dirotq_workspace_status(ws) == 0


def _prepared(fmt, W, Q, r=32):
    Uh = Q[:, :r].contiguous()
    return {"int4": lambda: dq.dirotq_prepare_layer(W, Q, r, 128), "int4_asym": lambda: dq.dirotq_prepare_layer_asym(W, Q, r, 64),
            "w4a8": lambda: dq.dirotq_prepare_layer_w4a8(W, Q, r), "nvfp4": lambda: dq.dirotq_prepare_layer_nvfp4(W, Q, r, -8),
            "int4_ph": lambda: dq.dirotq_prepare_layer_ph(W, Uh, 128), "nvfp4_ph": lambda: dq.dirotq_prepare_layer_nvfp4_ph(W, Uh, -8)}[fmt]()


@pytest.mark.parametrize("fmt", ["int4", "int4_asym", "w4a8", "nvfp4", "int4_ph", "nvfp4_ph"])
@pytest.mark.parametrize("M,hq,hk,D,rot,style", [(1, 4, 1, 128, 128, "halves"), (33, 6, 2, 72, 36, "halves"), (150, 5, 5, 96, 96, "pairs"), (700, 3, 1, 64, 0, None)])
def test_behind_prepared_layers(fmt, M, hq, hk, D, rot, style):
    K = 512
    s = Setup(M, hq, hk, D, rot, style, torch.bfloat16, M)
    g = _gen(3)
    W = 0.05 * torch.randn((K, s.width), device="cuda", generator=g)
    Q = torch.linalg.qr(torch.randn((K, K), dtype=torch.float64, device="cuda", generator=g))[0].contiguous()
    layer = _prepared(fmt, W, Q)
    x, ws = torch.randn((M, K), device="cuda", generator=g).bfloat16(), dq.alloc_workspace(layer, M)
    y, z = (torch.empty((M, s.width), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for _ in range(2):
        dq.dirotq_linear_qkv(x, layer, y, ws, s.plan)
    dq.dirotq_linear(x, layer, z, ws)
    assert dq.dirotq_workspace_status(ws) == 0
    nq, nk = hq * D, (hq + hk) * D
    (wq, tq), (wk, tk), _ = s.want(z)
    _within(y[:, :nq], wq, tq)
    _within(y[:, nq:nk], wk, tk)
    assert torch.equal(y[:, nk:], z[:, nk:])
    layer.close()
