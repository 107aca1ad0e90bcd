"""Memory that RolloutStack holds for the attention over an 8-bit cache: one workspace
for a whole rollout, whatever length the window has reached; smaller ones stay only
where a captured graph uses them."""
import pytest
import torch

import workloads as W

pytestmark = pytest.mark.gpu

HEADS, D, F, C, WINDOW = 10, 64, 700, 3, 12
BUDGETS = [W.HeadBudget(W.STATIC, 1, 11)] * 9 + [W.HeadBudget(W.DYNAMIC, 1, 0, 8, W.SCOPE_GLOBAL)]


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


def _stack():
    from paper_2605_09681_amd.layer import RolloutStack
    return RolloutStack(1, HEADS, D, F, WINDOW, C, F, cache="e4m3")


def _full(fkv, stack, n_q, n_cur):
    return fkv.fkv_chunk_attention_q8_workspace_size(stack.shape(WINDOW), fkv.make_heads(BUDGETS), n_q, n_cur)


def _rows(n, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((HEADS, n, D), generator=g).bfloat16().cuda() for _ in range(3)]


def test_a_window_that_fills_up(fkv):
    stack = _stack()
    Q, K, V = _rows(C * F)
    O = torch.empty_like(Q)
    full = _full(fkv, stack, C * F, C * F)
    assert full >= 2 * HEADS * WINDOW * F * D * 2          # the largest holds the copy
    before = torch.cuda.memory_allocated()
    for chunk in range(5):
        stack.run_layer(0, BUDGETS, W.ring_frame_slots(chunk, C, WINDOW).tolist(), Q, K, V, O)
        stack.append(0, K, V, W.chunk_write_slots(chunk, C, WINDOW).tolist())
        torch.cuda.synchronize()
        assert torch.cuda.memory_allocated() - before <= full + (1 << 20), chunk


def test_larger_calls_replace_it(fkv):
    """Growing calls free what they outgrow, also where another stream used it, but not under a captured graph."""
    stack = _stack()
    for s in range(0, WINDOW, C):
        _, K, V = _rows(C * F, s)
        stack.append(0, K, V, list(range(s, s + C)))
    slots = list(range(WINDOW))
    static = [W.HeadBudget(W.STATIC, 1, 11)] * HEADS

    def call(n, out, q):
        stack.run_layer(0, static, slots, q[0][:, :n].contiguous(), q[1][:, :n].contiguous(), q[2][:, :n].contiguous(), out)
    x = _rows(C * F, 50)
    small, big = (torch.empty((HEADS, n, D), dtype=torch.bfloat16, device="cuda") for n in (16, C * F))
    q = [t[:, :16].contiguous() for t in x]
    call(16, small, x)
    torch.cuda.synchronize()
    want = small.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stack.run_layer(0, static, slots, *q, small)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for n in (64, 300, 600, 1000):                     # each outgrows the last one
            out = torch.empty((HEADS, n, D), dtype=torch.bfloat16, device="cuda")
            call(n, out, x)
    torch.cuda.current_stream().wait_stream(side)
    call(C * F, big, x)
    torch.cuda.synchronize()
    junk = torch.full((1 << 22,), 0x7f, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        small.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(small, want)
    held = torch.cuda.memory_allocated()
    copy = big.clone()
    call(C * F, big, x)
    torch.cuda.synchronize()
    assert torch.equal(copy, big)
    del copy, junk
    sizes = [fkv.fkv_chunk_attention_q8_workspace_size(stack.shape(WINDOW), fkv.make_heads(static), n, n) for n in (16, C * F)]
    del stack, graph
    torch.cuda.synchronize()
    # what the stack held: its cache, the last workspace and the graph's own
    cache = 2 * HEADS * WINDOW * F * D + 2 * 4 * HEADS * WINDOW * 11
    assert held - torch.cuda.memory_allocated() <= cache + sum(sizes) + (1 << 22) + (1 << 22)
