"""Attention over an 8-bit cache where scores are far from zero: keys that weigh
nothing because their scores are the lowest there are, in whole pages and waves'
shares, and rows whose every score has a magnitude of 1e13 and more.  In place (in
parts, and one workgroup per query tile) and over the expanded copy."""
import math

import pytest
import torch

import workloads as W
from tests.cache8_ref import F32_STEP, attention_bounds, half_step
from test_gpu_cache8 import Attend, _budgets

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


# every query tile height (16 rows, 32, and 48 for d = 64), in parts and whole
IN_PLACE = [
    dict(heads=3, d=128, F=256, H=8, n_q=5, n_cur=200, budgets=_budgets(2, 1, 7, 8, W.SCOPE_GLOBAL)),
    dict(heads=3, d=64, F=300, H=13, L=100, n_q=1, n_cur=0, block=16, budgets=_budgets(2, 1, 11, 30, W.SCOPE_GLOBAL)),
    dict(heads=12, d=128, F=1300, H=5, n_q=81, n_cur=81, budgets=_budgets(6, 6, 5, 5, W.SCOPE_GLOBAL)),
    dict(heads=16, d=64, F=60, H=12, n_q=650, n_cur=130, budgets=_budgets(8, 8, 11, 9, W.SCOPE_GLOBAL)),
]
EXPANDED = [
    dict(heads=9, d=128, F=1560, H=8, n_q=1100, n_cur=1100, budgets=_budgets(5, 4, 8, 8, W.SCOPE_GLOBAL)),
    dict(heads=10, d=64, F=1500, L=500, H=9, n_q=1030, n_cur=200, budgets=_budgets(4, 6, 9, 20, W.SCOPE_GLOBAL)),
]
SIZES = [(s, w) for s in IN_PLACE for w in ("own", None)] + [(s, "own") for s in EXPANDED]
IDS = [f"d{s['d']}-q{s['n_q']}-cur{s['n_cur']}-F{s['F']}-{'parts' if w else 'whole'}" for s, w in SIZES]


def _fill(a, K):
    """The cache's keys, written by the library (their codes are tested elsewhere)."""
    s = a.shape
    V = torch.randn(K.shape, generator=torch.Generator().manual_seed(3))
    rows = [t.reshape(s.n_heads, -1, s.head_dim).to(torch.bfloat16).cuda() for t in (K, V)]
    a.fkv.fkv_append_frames_q8(s, None, None, *rows, list(range(s.cap_frames)), a.cache)


def _keys(a):
    """Random keys for every slot, [heads][cap][F][d]."""
    s = a.shape
    g = torch.Generator().manual_seed(4)
    return torch.randn((s.n_heads, s.cap_frames, s.frame_tokens, s.head_dim), generator=g)


@pytest.mark.parametrize("mask", [-1e30, -3.3895313892515355e38])
@pytest.mark.parametrize("size,workspace", SIZES, ids=IDS)
def test_keys_with_the_lowest_scores(fkv, size, workspace, mask):
    """Every third frame of the history, a run inside the others and most of the current tokens hold a large
    negative value (products that stay finite, or overflow to -infinity): their weight is 0, and a wave or a part
    that has no other keys adds nothing."""
    print(f"[gpu case] q8-lowest {size['d']} {size['n_q']} {workspace} {mask}", flush=True)
    a = Attend(fkv, **size)
    a.Q = (torch.rand(a.Q.shape, generator=torch.Generator().manual_seed(5)) + 0.5).bfloat16()   # one sign for every product
    K = 0.3 * _keys(a)
    K[:, a.slots[::3]] = mask                        # (clamped to 448 * 2^119 by the cache)
    F = a.shape.frame_tokens
    K[:, :, F // 3:F // 2] = mask
    _fill(a, K)
    n_cur = a.K_cur.shape[1]
    a.K_cur = (0.3 * a.K_cur.float()).bfloat16()
    a.K_cur[:, :n_cur - 5] = mask
    a.K_cur[:, n_cur - 2:] = mask
    O, lse = a.run(workspace)
    for h in range(a.shape.n_heads):
        k, v = a.sources(h)
        k, v = torch.cat([k, a.K_cur[h].double()]), torch.cat([v, a.V_cur[h].double()])
        live = k[:, 0] > -1e29                       # (the others' weights are 0 in 64 bits too)
        want, bound, wl, bl = attention_bounds(a.Q[h].double(), k[live], v[live], a.scale)
        assert bool(want.isfinite().all()) and bool(live.any())
        # (in blocks with a masked token every other code is 0: what is left of those keys is their share of the sum)
        assert bool(((O[h].cpu().double() - want).abs() <= bound).all()), h
        assert bool(((lse[h].cpu().double() - wl).abs() <= bl).all()), h


FAR = [(2.0 ** 40, None), (2.0 ** 100, None), (2.0 ** 117, 4.0)]


@pytest.mark.parametrize("far,scale", FAR, ids=["1e13", "1e31", "beyond-the-product"])
@pytest.mark.parametrize("size,workspace", SIZES, ids=IDS)
def test_every_score_is_far(fkv, size, workspace, far, scale):
    """Rows whose every score has a magnitude of 1e13 or more, positive or negative, next to ordinary rows.  A
    score is one exact product (channel 0 of the keys holds one of eight E4M3 values, the far queries are zero
    elsewhere), so the softmax is the mean over the keys that tie for the largest, whatever the magnitude: also
    where the score is finite and its product with the scale is not."""
    print(f"[gpu case] q8-far {size['d']} {size['n_q']} {workspace} {far}", flush=True)
    a = Attend(fkv, **size)
    if scale:
        a.scale = scale
    g = torch.Generator().manual_seed(6)
    levels = torch.tensor([448.0, 416.0, 384.0, 352.0, 320.0, 288.0, 256.0, 240.0])

    def level_of(shape):
        return levels[torch.randint(0, 8, shape, generator=g)]
    K = _keys(a)
    K[..., 0] = level_of(K.shape[:-1])               # every block's scale is 1: the levels are codes
    # one frame and the first current tokens lie below the others: whole pages without the maximum
    K[:, a.slots[0], :, 0] = 224.0
    _fill(a, K)
    a.K_cur = a.K_cur.clone()
    a.K_cur[:, :, 0] = level_of(a.K_cur.shape[:2]).bfloat16()
    a.K_cur[:, :64, 0] = 208.0
    a.Q[:, :, 0] = 0
    n_q = a.Q.shape[1]
    kind = torch.arange(n_q) % 3                     # 0: far above zero, 1: far below, 2: ordinary
    if n_q == 1:
        kind[0] = 1
    a.Q[:, kind < 2] = 0
    a.Q[:, kind == 0, 0] = far
    a.Q[:, kind == 1, 0] = -far
    O, lse = a.run(workspace)
    rows = kind < 2
    for h in range(a.shape.n_heads):
        k, v = a.sources(h)
        k, v = torch.cat([k, a.K_cur[h].double()]), torch.cat([v, a.V_cur[h].double()])
        q = a.Q[h].double()
        if not scale:
            want, bound, wl, bl = attention_bounds(q[~rows], k, v, a.scale)
            assert bool(((O[h].cpu().double()[~rows] - want).abs() <= bound).all()), h
            assert bool(((lse[h].cpu().double()[~rows] - wl).abs() <= bl).all()), h
        z = q[rows][:, :1] * k[:, 0] * a.scale       # exact up to the scale
        top = z.amax(1, keepdim=True)
        p = (z == top).double()
        n = p.sum(1, keepdim=True)
        want, mass = p @ v / n, p @ v.abs() / n
        # equal probabilities, rounded to bf16; sums in fp32, the output rounded once
        bound = half_step(torch.bfloat16) * 1.01 * (want.abs() + mass) + (k.shape[0] + 64) * 2 * F32_STEP * mass + 1e-30
        err = (O[h].cpu().double()[rows] - want).abs()
        assert bool((err <= bound).all()), (h, float((err / bound).max()))
        if not scale:                                # (beyond the product the logarithm has no fp32 value)
            wl = top[:, 0] + n[:, 0].log()
            # the product with the scale, its logarithm's base and the sum: at most eight half steps
            assert bool(((lse[h].cpu().double()[rows] - wl).abs() <= 8 * F32_STEP * wl.abs() + 1e-6).all()), h
