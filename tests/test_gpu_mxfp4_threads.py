"""Calls of all shapes from several host threads at once, each on a stream of its own, with weights that some of them share: the same bits as one at a time."""
import random
import threading

import pytest
import torch

from paper_2605_16732_b200 import binding as dq

pytestmark = pytest.mark.gpu
THREADS = 6


class Job:
    def __init__(self, g, M, K, hq, hk, D, style, kind, w):
        self.kind, width = kind, (hq + 2 * hk) * D
        self.x = torch.randn((M, K), device="cuda", generator=g).bfloat16()
        self.w = w or dq.dirotq_mxfp4_quantize(torch.randn((width, K), device="cuda", generator=g) * 0.05)
        angle = torch.rand((M, D // 2), device="cuda", generator=g) * 6
        self.qk, self.ws = dq.QkNorm(hq, hk, D, rope=style, cos=angle.cos(), sin=angle.sin()), dq.alloc_mxfp4_workspace(M, K)
        self.out = [torch.zeros((M, n), dtype=torch.bfloat16, device="cuda") for n in (width, hq * D, hk * D, hk * D)]

    def run(self):
        y, q, k, v = self.out
        if self.kind == "qkv":
            dq.dirotq_mxfp4_qkv(self.x, self.w, y, self.ws, self.qk)
            return
        dq.dirotq_mxfp4_linear(self.x, self.w, y, self.ws)
        if self.kind == "both":
            dq.dirotq_qk_norm_rope(y, self.qk, q, k, v)


def test_calls_from_several_threads():
    g, rng = torch.Generator(device="cuda").manual_seed(1), random.Random(5)
    shared = dq.dirotq_mxfp4_quantize(torch.randn((8 * 64, 512), device="cuda", generator=g) * 0.05)
    jobs = [Job(g, rng.choice((1, 2, 5, 8, 30, 64, 129, 300, 700, 1500)), rng.choice((256, 1152, 3000)), rng.choice((4, 9, 24)), rng.choice((1, 2, 5)), rng.choice((64, 128)),
                rng.choice(("pairs", "halves")), rng.choice(("linear", "qkv", "both")), None) for _ in range(3 * THREADS)]
    jobs += [Job(g, M, 512, 4, 2, 64, "pairs", kind, shared) for M, kind in zip((1, 16, 20, 100, 300, 900), ("linear", "qkv", "both") * 2)]
    want = []
    for j in jobs:
        j.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in j.out])
    errors, streams = [], [torch.cuda.Stream() for _ in range(THREADS)]

    def work(t):
        try:
            mine, r = jobs[t::THREADS], random.Random(t)
            with torch.cuda.stream(streams[t]):
                for j in mine + [r.choice(mine) for _ in range(100)]:
                    j.run()
        except BaseException as e:  # (to be seen by the test)
            errors.append(e)

    for _ in range(2):
        for j in jobs:
            for o in j.out:
                o.zero_()
        torch.cuda.synchronize()
        threads = [threading.Thread(target=work, args=(t,)) for t in range(THREADS)]
        [t.start() for t in threads]
        [t.join() for t in threads]
        torch.cuda.synchronize()
        assert not errors, errors
        for j, w in zip(jobs, want):
            assert all(torch.equal(o, v) for o, v in zip(j.out, w)), (j.x.shape, j.kind)
            assert dq.dirotq_workspace_status(j.ws) == 0
