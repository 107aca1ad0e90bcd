"""bf16 chunk attention of rows whose every score has a magnitude of 1e13 or more,
positive or negative, next to ordinary rows: over a compact copy and in place, under
every schedule.  A far row's score is one exact product (channel 0 of the keys holds
one of eight values, the query is zero elsewhere), so its softmax is the mean over
the keys that tie for the largest."""
import math

import pytest
import torch

from test_gpu_attn_edges import _check
from test_gpu_attn_redo import LQ, SCHEDULES, F, H, _Inputs

pytestmark = pytest.mark.gpu

LEVELS = torch.tensor([448.0, 416.0, 384.0, 352.0, 320.0, 288.0, 256.0, 240.0])
KIND = torch.arange(LQ) % 3                              # 0: far above zero, 1: far below, 2: ordinary


@pytest.mark.parametrize("schedule", SCHEDULES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("far", [2.0 ** 40, 2.0 ** 100])
def test_every_score_is_far(d, far, schedule):
    print(f"[gpu case] attention-far d={d} far={far} schedule={schedule}", flush=True)

    def queries(g, n):
        q = torch.randn(n, LQ, d, generator=g)
        q[:, :, 0] = 0
        q[:, KIND < 2] = 0
        q[:, KIND == 0, 0], q[:, KIND == 1, 0] = far, -far
        return q.bfloat16()

    def keys(g, n, kept):
        k = torch.randn(n, H * F + LQ, d, generator=g)
        k[:, :, 0] = LEVELS[torch.randint(0, 8, k.shape[:2], generator=g)]
        k[:, :F, 0] = 224.0                              # a frame and the last keys below the others
        k[:, -70:, 0] = 208.0
        k = k.bfloat16()
        return k[:, :H * F].contiguous(), k[:, H * F:].contiguous()

    x = _Inputs(schedule, d, d, keys, queries)
    O, lse = x.run()
    rows = KIND < 2
    for h, length in enumerate(x.lens):
        k = torch.cat([x.K[h, :length], x.Kq[h]]).double()
        v = torch.cat([x.V[h, :length], x.Vq[h]]).double()
        z = x.Q[h][rows, :1].double() * k[:, 0] / math.sqrt(d)
        top = z.amax(1, keepdim=True)
        p = (z == top).double()
        n = p.sum(1, keepdim=True)
        want, mass = p @ v / n, p @ v.abs() / n
        # equal probabilities, parts and outputs rounded to bf16 (half a step each); sums in fp32
        bound = 1.01 * 2.0 ** -8 * (2 * mass + want.abs()) + (k.shape[0] + 64) * 2.0 ** -23 * mass + 1e-30
        err = (O[h][rows] - want).abs()
        assert bool((err <= bound).all()), (h, float((err / bound).max()))
        wl = top[:, 0] + n[:, 0].log()
        assert bool(((lse[h][rows] - wl).abs() <= 8 * 2.0 ** -24 * wl.abs()).all()), h
    x.Q[:, rows] = 0                                     # the ordinary rows, as if the others were zero
    Ow, lw, bound, zmax = x.reference()
    O[:, rows], lse[:, rows] = Ow[:, rows], lw[:, rows]
    _check((O, lse), (Ow, lw, bound, zmax), zmax)
