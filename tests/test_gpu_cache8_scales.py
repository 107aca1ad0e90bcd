"""Readers of an 8-bit cache use a scale's exponent alone: a cache whose scales carry
other mantissas is scored, selected from and attended (in place and over the expanded
copy) as the one with the powers of two below them."""
import pytest
import torch

import workloads as W
from test_gpu_cache8 import Attend, _budgets, _cache, _shape

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


def _add_mantissas(cache):
    g = torch.Generator().manual_seed(9)
    for s in (cache.k_scale, cache.v_scale):
        s.mul_(1 + 0.99 * torch.rand(s.shape, generator=g).cuda())


@pytest.mark.parametrize("heads,d,F,H,L,block", [(3, 128, 130, 5, 65, 16), (2, 64, 333, 13, 111, 32), (2, 128, 1560, 3, 1560, 64)])
def test_scores(fkv, heads, d, F, H, L, block):
    shape = _shape(fkv, heads, d, F, H, H, 1, L)
    hs = fkv.make_heads(_budgets(0, heads, 0, 1, W.SCOPE_FRAME if L < F else W.SCOPE_GLOBAL))
    cache = _cache(fkv, shape, block, 61)
    K_cur = torch.randn((heads, F, d), generator=torch.Generator().manual_seed(62)).bfloat16().cuda()
    n_seg, out = fkv.fkv_num_segments(shape), []
    for _ in range(2):
        o = (torch.zeros((heads, n_seg), device="cuda"), torch.zeros((heads, n_seg), dtype=torch.int32, device="cuda"),
             torch.zeros(heads, dtype=torch.int32, device="cuda"))
        fkv.fkv_score_select_q8(shape, hs, cache, None, K_cur, *o)
        out.append(o)
        _add_mantissas(cache)
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("size", [
    dict(heads=3, d=128, F=100, H=5, L=25, n_q=16, n_cur=33, block=32, budgets=_budgets(1, 2, 2, 9, W.SCOPE_GLOBAL)),
    dict(heads=9, d=128, F=1560, H=8, n_q=1100, n_cur=1100, budgets=_budgets(5, 4, 8, 8, W.SCOPE_GLOBAL))], ids=["in-place", "expanded"])
def test_attention(fkv, size):
    a = Attend(fkv, **size)
    first = a.run()
    _add_mantissas(a.cache)
    assert all(torch.equal(x, y) for x, y in zip(a.run(), first))
