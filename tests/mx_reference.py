"""Plain 64-bit forms of the MXFP4 operators and of the norm and rotation of q and k, for the tests."""
import torch

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
FLOOR, CEIL = 0, 1


def quantize(x: torch.Tensor, rule: int = FLOOR):
    """x [rows, K] (cpu) -> codes uint8 [rows, K] (one per byte), scales uint8 [rows, ceil(K/32)]."""
    rows, K = x.shape
    x = x.double()
    sign = torch.signbit(x).to(torch.uint8) * 8
    codes = torch.empty((rows, K), dtype=torch.uint8)
    scales = torch.empty((rows, -(-K // 32)), dtype=torch.uint8)
    for j in range(scales.shape[1]):
        b = x[:, 32 * j:32 * j + 32]
        a = b.abs().amax(1)
        bad = ~torch.isfinite(b).all(1)
        _, e = torch.frexp(torch.where(bad | (a == 0), 1.0, a))  # a = m 2^e, m in [0.5, 1)
        e = e - 3                                                 # floor(log2 a) - 2
        if rule == CEIL:
            e = torch.where(a > 6 * torch.exp2(e.double()), e + 1, e)
        e = torch.where(a == 0, -127, e).clamp(min=-127)
        u = torch.where(bad[:, None], 0.0, b.abs()) / torch.exp2(e.double())[:, None]
        c = torch.zeros_like(u, dtype=torch.uint8)
        for i in range(7):
            mid = (LEVELS[i] + LEVELS[i + 1]) / 2
            c += ((u > mid) if i % 2 == 0 else (u >= mid)).to(torch.uint8)  # a tie goes to the even code
        codes[:, 32 * j:32 * j + 32] = torch.where(bad[:, None], 0, c + sign[:, 32 * j:32 * j + 32])
        scales[:, j] = torch.where(bad, 255, e + 127).to(torch.uint8)
    return codes, scales


def values(codes: torch.Tensor, scales: torch.Tensor) -> torch.Tensor:
    v = LEVELS.to(codes.device)[(codes & 7).long()]
    v = torch.where(codes > 7, -v, v)
    s = torch.where(scales == 255, float("nan"), torch.exp2(scales.double() - 127))
    return v * s.repeat_interleave(32, 1)[:, :codes.shape[1]]


def pack(codes: torch.Tensor) -> torch.Tensor:
    if codes.shape[1] % 2:
        codes = torch.nn.functional.pad(codes, (0, 1))
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).contiguous()


def unpack(packed: torch.Tensor, K: int) -> torch.Tensor:
    return torch.stack((packed & 15, packed >> 4), -1).flatten(1)[:, :K]


def product(a: torch.Tensor, b: torch.Tensor, bias=None):
    """(a b^T + bias, sum |a| |b|) in 64 bits."""
    y, mass = a @ b.T, a.abs() @ b.abs().T
    if bias is not None:
        y, mass = y + bias.double(), mass + bias.double().abs()
    return y, mass


def product_tolerance(y, mass, K: int, dtype):
    """Half a step of the stored type, and for the fp32 sums: the tensor core adds 64 products to the accumulator at a time, so an element
    sees ceil(K/64) additions (and the bias'), each off by at most 2^-22 of the sum of magnitudes (a truncated fp32 addition, 2^-23, of
    terms that were themselves aligned to the largest and truncated)."""
    f = torch.finfo(dtype)
    return y.abs() * f.eps / 2 + (-(-K // 64) + 1) * 2.0 ** -22 * (1 + f.eps) * mass + f.smallest_normal * f.eps / 2


def head(x, w, eps, cos, sin, style, rot, norm=True):
    """x [M, heads, D] in 64 bits; cos, sin [M, rot/2].  Returns the result and, per element, the magnitudes that went into it."""
    x = x.double()
    if norm:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
        if w is not None:
            x = x * w.double()
    mass = x.abs()
    if not style or rot == 0:
        return x, mass
    c, s = cos.double()[:, None], sin.double()[:, None]
    i = torch.arange(rot // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if style == "pairs" else (i, i + rot // 2)
    out, m = x.clone(), mass.clone()
    out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    m[..., a] = m[..., b] = mass[..., a] + mass[..., b]
    return out, m


def head_tolerance(y, mass, D: int, dtype):
    """Half a step of the stored type; the sum of D squares in fp32 (at most D additions, half of whose relative error reaches the root), two
    units in the last place of rsqrt, the two products by it and the weight, and the rotation's two products and addition."""
    f = torch.finfo(dtype)
    return y.abs() * f.eps / 2 + mass * (D / 2 + 10) * 2.0 ** -24 * (1 + f.eps) + f.smallest_normal * f.eps / 2
