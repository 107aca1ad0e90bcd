"""RolloutStack.run_layer over an 8-bit cache with a score row computed elsewhere, and
with other current tokens than the chunk's, or none."""
import pytest
import torch

import workloads as W
from tests.cache8_ref import attention_bounds, kept_tokens, values

pytestmark = pytest.mark.gpu

HEADS, D, F, C, WINDOW, L = 4, 64, 70, 2, 7, 35
BUDGETS = [W.HeadBudget(W.STATIC, 1, 2)] * 2 + [W.HeadBudget(W.DYNAMIC, 1, 0, 1, W.SCOPE_FRAME)] * 2
STATIC = [W.HeadBudget(W.STATIC, 1, 2)] * HEADS
SLOTS = [3, 0, 5, 1, 2, 6]


@pytest.fixture(scope="module")
def stack():
    from paper_2605_09681_amd.layer import RolloutStack
    s = RolloutStack(2, HEADS, D, F, WINDOW, C, L, cache="e4m3", block_tokens=32)
    g = torch.Generator().manual_seed(1)
    for layer in range(2):
        K, V = (torch.randn((HEADS, WINDOW * F, D), generator=g).bfloat16().cuda() for _ in range(2))
        s.append(layer, K, V, list(range(WINDOW)))
    return s


def _rows(n, seed):
    return torch.randn((HEADS, n, D), generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def _check(stack, layer, budgets, Q, K, V, O, lse):
    c8 = stack.cache8[layer]
    Kc, Vc = values(c8.K.cpu(), c8.k_scale.cpu(), 32), values(c8.V.cpu(), c8.v_scale.cpu(), 32)
    kept, kv = stack.views(len(SLOTS))[1].cpu().numpy(), stack.kv_len.cpu().numpy()
    for h in range(HEADS):
        tok = kept_tokens(h, budgets, kept, kv, len(SLOTS), F, L)
        k, v = (x[h][SLOTS].reshape(-1, D)[tok] for x in (Kc, Vc))
        if K is not None:
            k, v = torch.cat([k, K[h].cpu().double()]), torch.cat([v, V[h].cpu().double()])
        want, bound, wl, bl = attention_bounds(Q[h].cpu().double(), k, v, stack.scale)
        assert bool(((O[h].cpu().double() - want).abs() <= bound).all()), h
        assert bool(((lse[h].cpu().double() - wl).abs() <= bl).all()), h


@pytest.mark.parametrize("n_q,n_cur", [(C * F, C * F), (1, 9), (5, 0), (3, None)])
def test_a_pooled_row(stack, n_q, n_cur):
    """The row selects in every layer, whatever the current tokens."""
    n_seg = 2 * len(SLOTS)
    row = torch.rand(n_seg, generator=torch.Generator().manual_seed(2)).cuda()
    for layer in range(2):
        Q = _rows(n_q, 3)
        K, V = (None, None) if n_cur is None else (_rows(n_cur, 4), _rows(n_cur, 5))
        O, lse = torch.empty_like(Q), torch.empty((HEADS, n_q), device="cuda")
        stack.run_layer(layer, BUDGETS, SLOTS, Q, K, V, O, lse, pooled=row)
        kept = stack.views(len(SLOTS))[1].cpu()
        least = [0, 1] + [2 * t + int(row[2 * t + 1] < row[2 * t]) for t in range(1, len(SLOTS))]
        for h in (2, 3):
            assert kept[h].tolist()[:len(least)] == least and stack.kv_len[h] == len(least) * L
        _check(stack, layer, BUDGETS, Q, K, V, O, lse)


@pytest.mark.parametrize("n_cur", [None, 0, 3, 200])
def test_static_heads_with_other_current_tokens(stack, n_cur):
    Q = _rows(7, 6)
    K, V = (None, None) if n_cur is None else (_rows(n_cur, 7), _rows(n_cur, 8))
    O, lse = torch.empty_like(Q), torch.empty((HEADS, 7), device="cuda")
    stack.run_layer(0, STATIC, SLOTS, Q, K, V, O, lse)
    _check(stack, 0, STATIC, Q, K, V, O, lse)


def test_scoring_needs_the_chunk(stack):
    Q = _rows(7, 9)
    O = torch.empty_like(Q)
    with pytest.raises(ValueError):
        stack.run_layer(0, BUDGETS, SLOTS, Q, None, None, O)
    with pytest.raises(ValueError):
        stack.run_layer(0, BUDGETS, SLOTS, Q, _rows(9, 1), _rows(9, 2), O)
