"""Paths of the 8-bit cache's calls that sizes alone select: long histories in the
scoring, large chunks whose current tokens are fewer or more than the queries, and
large chunks whose segments are computed again with a running maximum."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from tests.cache8_ref import F32_STEP, attention_bounds, values
from test_gpu_cache8 import Attend, _budgets, _cache, _shape

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("heads,d,F,H,L,block", [
    (2, 128, 24, 24, 24, 16), (2, 64, 24, 25, 24, 16), (2, 64, 30, 47, 10, 32), (2, 128, 8, 64, 32, 64), (1, 64, 3, 200, 3, 16)])
def test_scores_of_long_histories(fkv, heads, d, F, H, L, block):
    """Histories of more frames than a wave holds at once, within the bound that fkv.h states; the selection is that
    of the bf16 cache of the same values."""
    shape = _shape(fkv, heads, d, F, H, H, 1, L)
    scope = W.SCOPE_FRAME if L < F else W.SCOPE_GLOBAL
    hs = fkv.make_heads(_budgets(0, heads, 0, 2 if L < F else H // 2, scope))
    cache = _cache(fkv, shape, block, 51)
    slots = np.random.default_rng(52).permutation(H).tolist()
    K_cur = torch.randn((heads, F, d), generator=torch.Generator().manual_seed(53)).bfloat16().cuda()
    n_seg = fkv.fkv_num_segments(shape)
    out = [(torch.zeros((heads, n_seg), device="cuda"), torch.zeros((heads, n_seg), dtype=torch.int32, device="cuda"),
            torch.zeros(heads, dtype=torch.int32, device="cuda")) for _ in range(2)]
    fkv.fkv_score_select_q8(shape, hs, cache, slots, K_cur, *out[0])
    val = values(cache.K.cpu(), cache.k_scale.cpu(), block)
    fkv.fkv_score_select(shape, hs, val.bfloat16().cuda(), slots, K_cur, *out[1])
    assert torch.equal(out[0][1], out[1][1]) and torch.equal(out[0][2], out[1][2])
    seq = torch.cat([val[:, slots].reshape(heads, H * F, d), K_cur.cpu().double()], 1)
    for g in range(n_seg):
        lo, hi = g * L, min(g * L + L, H * F)
        u, w = seq[:, lo:hi].flatten(1), seq[:, lo + F:hi + F].flatten(1)
        c = (u * w).sum(1) / ((u * u).sum(1) * (w * w).sum(1)).sqrt()
        assert bool(((out[0][0].cpu().double()[:, g] - c).abs() <= F32_STEP * c.abs() + (3 + 3 * c.abs()) * F32_STEP).all())


@pytest.mark.parametrize("d,F,n_q,n_cur", [(128, 1560, 1100, 37), (128, 1560, 700, 2500), (64, 1500, 1500, 1)])
def test_expanded_chunks_with_other_current_tokens(fkv, d, F, n_q, n_cur):
    a = Attend(fkv, heads=12, d=d, F=F, H=8, n_q=n_q, n_cur=n_cur, budgets=_budgets(6, 6, 8, 8, W.SCOPE_GLOBAL))
    n = fkv.fkv_chunk_attention_q8_workspace_size(a.shape, a.heads, n_q, n_cur)
    assert n >= 2 * 12 * 2 * d * F * 8                # it holds the copy: this call takes that way
    a.check(*a.run())


EXPANDED = [dict(heads=12, d=128, F=1000, H=8, n_q=1300, n_cur=1300, budgets=_budgets(6, 6, 8, 8, W.SCOPE_GLOBAL)),
            dict(heads=10, d=64, F=1500, L=500, H=9, n_q=1030, n_cur=150, budgets=_budgets(4, 6, 9, 20, W.SCOPE_GLOBAL))]


def _levels(a, span):
    """Keys and queries whose frames, and runs of 64 current tokens, have levels of scores of their own, `span`
    nats apart at most."""
    s, g = a.shape, torch.Generator().manual_seed(7)
    d = s.head_dim
    u = torch.ones(d) / math.sqrt(d)
    a.Q = (torch.randn(a.Q.shape, generator=g) * 0.5 + 4 * u).bfloat16()
    n_cur = a.K_cur.shape[1]
    hist = torch.rand((s.n_heads, s.cap_frames, 1, 1), generator=g) * span
    cur = (torch.rand((s.n_heads, -(-n_cur // 64)), generator=g) * span).repeat_interleave(64, 1)[:, :n_cur, None]
    cur[:, -64:] = 0
    K = torch.randn((s.n_heads, s.cap_frames, s.frame_tokens, d), generator=g) * 0.5 + hist / (4 * a.scale) * u
    a.K_cur = (torch.randn((s.n_heads, n_cur, d), generator=g) * 0.5 + cur / (4 * a.scale) * u).bfloat16()
    V = torch.randn(K.shape, generator=g)
    rows = [t.reshape(s.n_heads, -1, d).bfloat16().cuda() for t in (K, V)]
    a.fkv.fkv_append_frames_q8(s, None, None, *rows, list(range(s.cap_frames)), a.cache)


@pytest.mark.parametrize("span", [40.0, 90.0, 400.0])
@pytest.mark.parametrize("size", EXPANDED, ids=["d128", "d64"])
def test_expanded_levels(fkv, size, span):
    """Sums of up to 2^57, above 2^100 and beyond the fp32 range against the first tile's maximum."""
    print(f"[gpu case] q8-levels {size['d']} {span}", flush=True)
    a = Attend(fkv, **size)
    _levels(a, span)
    a.check(*a.run())
    a.check(*a.run(workspace=None))


@pytest.mark.parametrize("size", EXPANDED, ids=["d128", "d64"])
def test_expanded_not_finite(fkv, size):
    """A NaN code, an infinite value and a NaN query reach what they weigh in and nothing else."""
    a = Attend(fkv, **size)
    O0, l0 = a.run()
    a.cache.V.view(torch.uint8)[0, a.slots[-1], 11, 5] = 0x7f
    a.V_cur[1, 9, 7] = math.inf
    a.Q[2, 5, 0] = math.nan
    O, lse = a.run()
    bad = torch.zeros(O.shape, dtype=torch.bool, device="cuda")
    bad[0, :, 5] = bad[1, :, 7] = bad[2, 5] = True
    assert bool(O[0, :, 5].isnan().all()) and bool((O[1, :, 7] == math.inf).all())
    assert bool(O[2, 5].isnan().all()) and bool(lse[2, 5].isnan())
    a.Q[2, 5, 0] = 0
    a.cache.V.view(torch.uint8)[0, a.slots[-1], 11, 5] = 0
    a.V_cur[1, 9, 7] = 0
    for h in range(3):
        k, v = a.sources(h)
        k, v = torch.cat([k, a.K_cur[h].double()]), torch.cat([v, a.V_cur[h].double()])
        want, bound, wl, bl = attention_bounds(a.Q[h].double(), k, v, a.scale)
        ok = ~bad[h].cpu()
        assert bool(((O[h].cpu().double() - want).abs() <= bound)[ok].all()), h
        assert bool(((lse[h].cpu().double() - wl).abs() <= bl)[ok[:, 0]].all()), h
