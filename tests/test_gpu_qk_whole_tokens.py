"""Norm and rotation of q and k where a warp takes all of a token's heads, set after set (many tokens), in every style of rotation and type: out of place
with v, in place, and by slots with padding tokens.  Head counts that are and are not whole sets."""
import pytest
import torch

from paper_2605_16732_b200 import binding as dq
from test_gpu_qk_norm import Setup, _gen, _within

pytestmark = pytest.mark.gpu
M = 2500  # (from 16 tokens per SM on)
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
CASES = [  # q heads, kv heads, head_dim, rotated, style; in 16 bits a set is 8 heads of 128, 12 of 72, 16 of 64, half as many in 32 bits
    (24, 24, 128, 128, "pairs"), (24, 9, 128, 128, "halves"), (16, 16, 72, 36, "halves"), (29, 13, 72, 72, "pairs"), (20, 9, 128, 48, "halves"),
    (20, 20, 128, 0, None), (17, 17, 128, 64, "halves"), (33, 16, 64, 32, "pairs"), (50, 17, 64, 64, "halves"), (40, 40, 96, 0, None), (11, 7, 160, 160, "pairs"),
    (19, 5, 96, 48, "halves"), (9, 9, 256, 256, "halves"), (13, 12, 80, 30, "halves")]


@pytest.mark.parametrize("hq,hk,D,rot,style", CASES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_out_of_place_and_in_place(hq, hk, D, rot, style, dtype):
    s = Setup(M, hq, hk, D, rot, style, dtype, D + rot)
    q, k, v = (torch.empty((M, n * D), dtype=dtype, device="cuda") for n in (hq, hk, hk))
    before = s.x.clone()
    dq.dirotq_qk_norm_rope(s.x, s.plan, q, k, v)
    (wq, tq), (wk, tk), wv = s.want()
    _within(q, wq, tq)
    _within(k, wk, tk)
    assert torch.equal(v.double(), wv) and torch.equal(s.x, before)
    y = s.x.clone()
    nq, nk = hq * D, (hq + hk) * D
    dq.dirotq_qk_norm_rope(y, s.plan, y[:, :nq], y[:, nq:nk])
    assert torch.equal(y[:, :nq], q) and torch.equal(y[:, nq:nk], k) and torch.equal(y[:, nk:], before[:, nk:])


@pytest.mark.parametrize("hq,hk,D,rot,style", [(24, 24, 128, 128, "pairs"), (25, 17, 72, 36, "halves"), (20, 9, 128, 48, "halves"), (33, 33, 64, 64, "halves")])
@pytest.mark.parametrize("dtype", DTYPES)
def test_slots_and_padding(hq, hk, D, rot, style, dtype):
    s = Setup(M, hq, hk, D, rot, style, dtype, D)
    rows = M + 300
    slots = torch.randperm(rows, device="cuda", generator=_gen(9))[:M].to(torch.int32)
    slots[::11], slots[5::97] = -1, rows
    s.positions[3::13], s.positions[7::101] = -1, len(s.cos)
    q = torch.full((M, hq * D), 5, dtype=dtype, device="cuda")
    cache = torch.full((rows, 2, hk * D + 8), 5, dtype=dtype, device="cuda")
    dq.dirotq_qk_norm_rope(s.x, s.plan, q, cache[:, 0, :hk * D], cache[:, 1, :hk * D], slots=slots)
    (wq, tq), (wk, tk), wv = s.want()
    live = (slots >= 0) & (slots < rows) & (s.positions >= 0) & (s.positions < len(s.cos))
    assert 0 < int(live.sum()) < M
    _within(q[live], wq[live], tq[live])
    at = slots[live].long()
    _within(cache[at, 0, :hk * D], wk[live], tk[live])
    assert torch.equal(cache[at, 1, :hk * D].double(), wv[live])
    others = torch.ones(rows, dtype=torch.bool, device="cuda")
    others[at] = False
    assert bool((cache[others] == 5).all()) and bool((cache[:, :, hk * D:] == 5).all()) and bool((q[~live] == 5).all())


@pytest.mark.parametrize("D,rot,style", [(128, 128, "pairs"), (72, 36, "halves"), (128, 48, "halves"), (64, 0, None)])
def test_a_tokens_bits_do_not_depend_on_the_other_tokens(D, rot, style):
    hq, hk = 21, 10
    s = Setup(M, hq, hk, D, rot, style, torch.bfloat16, 3, positions=False)
    q, k, v = (torch.empty((M, n * D), dtype=torch.bfloat16, device="cuda") for n in (hq, hk, hk))
    dq.dirotq_qk_norm_rope(s.x, s.plan, q, k, v)
    for m in (1, 100, 2300):
        qq, kk, vv = (torch.empty((m, n * D), dtype=torch.bfloat16, device="cuda") for n in (hq, hk, hk))
        dq.dirotq_qk_norm_rope(s.x[:m], s.plan, qq, kk, vv)
        assert torch.equal(qq, q[:m]) and torch.equal(kk, k[:m]) and torch.equal(vv, v[:m])
