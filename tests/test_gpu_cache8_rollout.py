"""RolloutStack with positions and with an 8-bit cache: whole rollouts across the
ring's wrap (rotate, score and select, attend, append), every step against plain
forms in 64 bits over what the cache holds, and the cache against the rotated and
quantised frames."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from tests.cache8_ref import (E4M3, Rope, attention_bounds, half_step, kept_tokens, rotate64, rotation_slack, values)

pytestmark = pytest.mark.gpu

HEADS, D, F, C, WINDOW, L = 4, 64, 70, 2, 7, 35
BUDGETS = [W.HeadBudget(W.STATIC, 1, 2)] * 2 + [W.HeadBudget(W.DYNAMIC, 1, 0, 1, W.SCOPE_FRAME)] * 2


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


def _stack(fkv, **kw):
    from paper_2605_09681_amd.layer import RolloutStack
    return RolloutStack(2, HEADS, D, F, WINDOW, C, L, **kw)


def _chunk(seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((C * F, 3, HEADS, D), generator=g).to(torch.bfloat16).cuda()
    return [x[:, i].transpose(0, 1) for i in range(3)]


def _buffers():
    return [torch.empty((HEADS, C * F, D), dtype=torch.bfloat16, device="cuda") for _ in range(4)]


ROPE = Rope(12, 10, 10, row_tokens=10)


def test_rollout_in_8_bits(fkv):
    stack = _stack(fkv, cache="e4m3", block_tokens=32, rope=ROPE.make(fkv))
    held = {}                                         # (layer, slot) -> the frame's rotated keys and its values, 64 bits
    lse = torch.empty((HEADS, C * F), device="cuda")
    for chunk in range(6):
        slots = W.ring_frame_slots(chunk, C, WINDOW).tolist()
        pos = [chunk * C + f for f in range(C)]
        H = len(slots)
        for layer in range(2):
            Q, K, V = _chunk(100 * chunk + layer)
            Qr, Kr, Vr, O = _buffers()
            stack.rotate(pos, Q, K, V, Qr, Kr, Vr)
            stack.run_layer(layer, BUDGETS, slots, Qr, Kr, Vr, O, lse)
            _, kept = stack.views(H)
            kept, kv = kept.cpu().numpy(), stack.kv_len.cpu().numpy()
            c8 = stack.cache8[layer]
            Kc, Vc = values(c8.K.cpu(), c8.k_scale.cpu(), 32), values(c8.V.cpu(), c8.v_scale.cpu(), 32)
            for s in slots:                           # the cache holds what was appended
                for got, want, slack, scale in ((Kc, *held[layer, s][0], c8.k_scale), (Vc, *held[layer, s][1], c8.v_scale)):
                    unit = scale.cpu()[:, s].double().repeat_interleave(32, -1)[:, :F, None]
                    bound = torch.maximum(half_step(E4M3) * want.abs(), unit * 2.0 ** -10) + 1.07 * slack
                    assert bool(((got[:, s] - want).abs() <= bound).all())
            for h in range(HEADS):
                tok = kept_tokens(h, BUDGETS, kept, kv, H, F, L)
                k = Kc[h][slots].reshape(-1, D)[tok]
                v = Vc[h][slots].reshape(-1, D)[tok]
                if BUDGETS[h].type == W.DYNAMIC and H > 1:
                    assert len(tok) == F + (H - 1) * L
                want, bound, wl, bl = attention_bounds(Qr[h].cpu().double(), torch.cat([k, Kr[h].cpu().double()]),
                                                       torch.cat([v, Vr[h].cpu().double()]), stack.scale)
                assert bool(((O[h].cpu().double() - want).abs() <= bound).all())
                assert bool(((lse[h].cpu().double() - wl).abs() <= bl).all())
            # one query token over the same cache, no lse
            one = torch.empty((HEADS, 1, D), dtype=torch.bfloat16, device="cuda")
            stack.run_layer(layer, BUDGETS, slots, Qr[:, 3:4].contiguous(), Kr, Vr, one)
            assert float((one[:, 0].float() - O[:, 3].float()).abs().max()) <= 2 * float(bound.max()) + 2 ** -8
            dst = W.chunk_write_slots(chunk, C, WINDOW).tolist()
            stack.append(layer, K, V, dst, frame_pos=pos)
            turned, slack = rotate64(K.cpu(), ROPE, pos, F), rotation_slack(K.cpu(), ROPE)
            for f, s in enumerate(dst):
                rows = slice(f * F, f * F + F)
                held[layer, s] = ((turned[:, rows], slack[:, rows]), (V.cpu().double()[:, rows], 0.0))


def test_rollout_with_positions_in_bf16(fkv):
    """append(frame_pos) writes the bits that rotate() gives, and the other slots stay."""
    stack = _stack(fkv, rope=ROPE.make(fkv))
    other = _stack(fkv)
    for chunk in range(5):
        Q, K, V = _chunk(chunk)
        Qr, Kr, Vr, _ = _buffers()
        pos = [chunk * C + f for f in range(C)]
        stack.rotate(pos, Q, K, V, Qr, Kr, Vr)
        dst = W.chunk_write_slots(chunk, C, WINDOW).tolist()
        stack.append(0, K, V, dst, frame_pos=pos)
        other.append(0, Kr, Vr, dst)
        assert torch.equal(stack.K_hist[0], other.K_hist[0]) and torch.equal(stack.V_hist[0], other.V_hist[0])
        assert not bool(stack.K_hist[1].any())


def test_graph_keeps_its_workspace(fkv):
    """A captured step replays right after larger eager calls have grown the stack's workspace."""
    stack = _stack(fkv, cache="e4m3")
    static = [W.HeadBudget(W.STATIC, 0, WINDOW)] * HEADS
    for s in range(WINDOW // 2):
        _, K, V = _chunk(s)
        stack.append(0, K, V, [2 * s, 2 * s + 1])
    slots = list(range(6))
    Q, K, V = (t.contiguous() for t in _chunk(50))
    q, k, v = Q[:, :1].contiguous(), K[:, :5].contiguous(), V[:, :5].contiguous()
    O = torch.empty_like(q)
    stack.run_layer(0, static, slots, q, k, v, O)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stack.run_layer(0, static, slots, q, k, v, O)
    big = torch.empty_like(Q)
    for seed in range(3):
        q.copy_(_chunk(60 + seed)[0][:, :1])
        graph.replay()
        got = O.clone()
        stack.run_layer(0, static, slots, Q, K, V, big)
        junk = torch.full((1 << 20,), 0x7f, dtype=torch.uint8, device="cuda")       # memory that a freed workspace would be
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, got)
        stack.run_layer(0, static, slots, q, k, v, O)
        assert torch.equal(O, got)
        del junk


def test_refusals(fkv):
    for kw in (dict(cache="int4"), dict(cache="e4m3", dtype="f32"), dict(cache="e4m3", step_mode="paged"),
               dict(cache="e4m3", block_tokens=24)):
        with pytest.raises(ValueError):
            stack = _stack(fkv, **kw)
            stack.append(0, *_chunk(0)[1:], [0, 1])
    stack = _stack(fkv, cache="e4m3")
    Q, K, V = (t.contiguous() for t in _chunk(0))
    with pytest.raises(ValueError):
        stack.append(0, K, V, [0, 1], frame_pos=[0, 1])          # no rope
    with pytest.raises(ValueError):
        stack.rotate([0, 1], Q, K, V, Q, K, V)
    with pytest.raises(ValueError):
        stack.history(0, BUDGETS, [0])
    with pytest.raises(ValueError):
        stack.score_pooled(0, [0], K)
    with pytest.raises(ValueError):
        stack.run_layer(0, BUDGETS, [0], Q, K, V, Q.clone(), incremental=True)
