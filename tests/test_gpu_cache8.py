"""Position rotation, appending with rotation, and the 8-bit rolling cache on the
GPU, against plain forms in 64 bits (tests/cache8_ref.py) at the sizes, strides,
budgets and values where they can go wrong.  Tolerances are bounds of the
arithmetic: one rounding to the output's type, and the stated bounds of the fp32
steps before it."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from tests.cache8_ref import (E4M3, F32_STEP, Rope, attention_bounds, exponent_of, half_step, kept_tokens, quantise,
                              rotate64, rotation_slack, values)

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


def _shape(fkv, heads=2, d=128, F=64, H=4, cap=None, C=1, L=None, dtype="bf16"):
    return fkv.make_shape(heads, d, F, H, H if cap is None else cap, C, F if L is None else L, dtype)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _projection(g, n, heads, d, dtype):
    """Q, K, V as views of one [n][3][heads][d] projection."""
    x = torch.randn((n, 3, heads, d), generator=g).to(DT[dtype]).cuda()
    return [x[:, i].transpose(0, 1) for i in range(3)]


ROPES = [
    ("video", dict(frame_pairs=22, row_pairs=21, col_pairs=21, row_tokens=13)),
    ("sequence", dict(frame_pairs=32, token_step=1, halves=True)),
    ("partial", dict(frame_pairs=5, col_pairs=7, row_tokens=4, theta=500.0, halves=True)),
    ("rows", dict(frame_pairs=0, row_pairs=16, row_tokens=1)),
    ("none", dict(frame_pairs=0)),
]


def _rope(name, d, F):
    kw = dict(next(r for n, r in ROPES if n == name))
    if d == 64:
        kw = {k: v // 2 if k.endswith("_pairs") else v for k, v in kw.items()}
    kw["row_tokens"] = min(kw.get("row_tokens", 1), F)
    return Rope(**kw)


def _check_rotated(got, x, rope, pos, F):
    want = rotate64(x.cpu(), rope, pos, F)
    err = (got.cpu().double() - want).abs()
    bound = half_step(got.dtype) * want.abs() + rotation_slack(x.cpu(), rope)
    assert bool((err <= bound).all()), float((err / bound.clamp(min=1e-300)).max())


@pytest.mark.parametrize("name", [n for n, _ in ROPES])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,d,F,C", [(3, 128, 65, 2), (5, 64, 7, 3), (1, 128, 1, 1), (2, 64, 1, 2)])
def test_rotate_chunk(fkv, name, dtype, heads, d, F, C):
    rope = _rope(name, d, F)
    shape = _shape(fkv, heads, d, F, 1, 4, C, dtype=dtype)
    Q, K, V = _projection(_gen(1), C * F, heads, d, dtype)
    pos = [17 + 3 * f for f in range(C)]
    out = [torch.full((heads, C * F, d), 7.0, dtype=DT[dtype], device="cuda") for _ in range(3)]
    fkv.fkv_rotate_chunk(shape, rope.make(fkv), pos, Q, K, V, *out)
    _check_rotated(out[0], Q, rope, pos, F)
    _check_rotated(out[1], K, rope, pos, F)
    assert torch.equal(out[2], V)
    # the keys alone, from a contiguous tensor and in place: the same bits
    alone = K.contiguous()
    fkv.fkv_rotate_chunk(shape, rope.make(fkv), pos, None, alone, None, None, alone, None)
    assert torch.equal(alone, out[1])


@pytest.mark.parametrize("pos", [0, -5, 1 << 24, -(1 << 24), 9999991])
def test_far_positions(fkv, pos):
    rope = Rope(32, 16, 16, row_tokens=5)
    shape = _shape(fkv, 2, 128, 33, 1, 1, 1, dtype="f32")
    Q, K, _ = _projection(_gen(2), 33, 2, 128, "f32")
    out = [torch.empty((2, 33, 128), device="cuda") for _ in range(2)]
    fkv.fkv_rotate_chunk(shape, rope.make(fkv), [pos], Q, K, None, out[0], out[1], None)
    _check_rotated(out[0], Q, rope, [pos], 33)
    _check_rotated(out[1], K, rope, [pos], 33)


def test_rotation_keeps_what_is_not_finite_in_its_pair(fkv):
    """An infinity or a NaN spoils its own pair and no other channel."""
    rope = Rope(64)
    shape = _shape(fkv, 1, 128, 4, 1, 1, 1)
    x = torch.randn((1, 4, 128), generator=_gen(3)).to(torch.bfloat16)
    clean = rotate64(x, rope, [3], 4)
    x[0, 1, 10], x[0, 2, 20] = math.inf, math.nan
    out = torch.empty_like(x).cuda()
    fkv.fkv_rotate_chunk(shape, rope.make(fkv), [3], x.cuda(), None, None, out, None, None)
    out = out.cpu().double()
    bad = torch.zeros(4, 128, dtype=torch.bool)
    bad[1, 10:12] = bad[2, 20:22] = True
    assert not bool(torch.isfinite(out[0][bad]).any())
    assert bool(((out[0] - clean[0]).abs()[~bad] <= (half_step(torch.bfloat16) * clean[0].abs() + 1e-5)[~bad]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,d,F,n,cap", [(3, 128, 65, 2, 5), (17, 64, 3, 1, 1), (2, 128, 1, 4, 6)])
def test_append_rotated(fkv, dtype, heads, d, F, n, cap):
    rope = _rope("video", d, F)
    shape = _shape(fkv, heads, d, F, 0, cap, 1, dtype=dtype)
    _, K, V = _projection(_gen(4), n * F, heads, d, dtype)
    slots = np.random.default_rng(1).permutation(cap)[:n].tolist()
    pos = [100 + f for f in range(n)]
    Kh = torch.full((heads, cap, F, d), 3.0, dtype=DT[dtype], device="cuda")
    Vh = torch.full_like(Kh, 4.0)
    fkv.fkv_append_frames_rotated(shape, rope.make(fkv), pos, K, V, slots, Kh, Vh)
    _check_rotated(Kh[:, slots].reshape(heads, n * F, d), K, rope, pos, F)
    assert torch.equal(Vh[:, slots].reshape(heads, n * F, d), V)
    others = [s for s in range(cap) if s not in slots]
    assert bool((Kh[:, others] == 3).all()) and bool((Vh[:, others] == 4).all())


# ------------------------------------------------------------ the 8-bit cache
def _block_values(g, heads, n, F, d):
    """Rows whose blocks have unlike sizes, among them zeros, borders of the scale and its ends."""
    x = torch.randn((heads, n, F, d), generator=g)
    x *= torch.exp(3 * torch.randn((heads, n, F, 1), generator=g))
    x[0, 0, 0] = 0
    x[0, 0, F // 2, 1] = 448.0 * 8
    x[-1, -1, F - 1, :] = 2.0 ** -120
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("heads,d,F,n", [(3, 128, 130, 2), (2, 64, 65, 1), (5, 128, 1, 2), (13, 64, 16, 1)])
def test_append_q8_codes(fkv, dtype, block, heads, d, F, n):
    """Without a rotation the codes and scales are exactly the definition's."""
    cap = n + 2
    shape = _shape(fkv, heads, d, F, 0, cap, 1, dtype=dtype)
    g = _gen(5)
    K, V = (_block_values(g, heads, n, F, d).to(DT[dtype]) for _ in range(2))
    cache = fkv.Cache8.zeros(shape, block)
    for t in (cache.K, cache.V):
        t.view(torch.uint8).fill_(0x3a)
    cache.k_scale.fill_(0.5)
    cache.v_scale.fill_(0.25)
    slots = list(range(cap))[::-1][:n]
    fkv.fkv_append_frames_q8(shape, None, None, K.reshape(heads, n * F, d).cuda(), V.reshape(heads, n * F, d).cuda(),
                             slots, cache)
    for x, codes, scales, rest in ((K, cache.K, cache.k_scale, 0.5), (V, cache.V, cache.v_scale, 0.25)):
        want, ws = quantise(x.float(), block)
        assert torch.equal(scales.cpu()[:, slots], ws)
        assert torch.equal(codes.cpu().view(torch.uint8)[:, slots], want.view(torch.uint8))
        others = [s for s in range(cap) if s not in slots]
        assert bool((codes.view(torch.uint8)[:, others] == 0x3a).all()) and bool((scales[:, others] == rest).all())


@pytest.mark.parametrize("amax", [448.0, 449.0, 2.0 ** 119 * 448, 3.0e38, 2.0 ** -92, 1e-38, 1e-45, 240.0, 256.0])
def test_append_q8_scale_borders(fkv, amax):
    shape = _shape(fkv, 1, 64, 16, 0, 1, 1, dtype="f32")
    x = torch.zeros((1, 16, 64))
    x[0, 3, 5] = -amax
    x[0, 2, 1] = amax / 3
    cache = fkv.Cache8.zeros(shape, 16)
    fkv.fkv_append_frames_q8(shape, None, None, x.cuda(), x.cuda(), [0], cache)
    want, ws = quantise(x[:, None], 16)
    assert torch.equal(cache.k_scale.cpu(), ws) and torch.equal(cache.v_scale.cpu(), ws)
    assert torch.equal(cache.K.cpu().view(torch.uint8), want.view(torch.uint8))
    assert float(ws[0, 0, 0]) == 2.0 ** exponent_of(float(torch.tensor(amax)))


def test_append_q8_not_finite(fkv):
    """Infinities and NaN become NaN; the block's scale and other codes are those without them."""
    shape = _shape(fkv, 2, 128, 40, 0, 1, 1)
    x = torch.randn((2, 40, 128), generator=_gen(6)).to(torch.bfloat16)
    bad = torch.zeros(x.shape, dtype=torch.bool)
    bad[0, 3, 7] = bad[0, 20, 1] = bad[1, 39, 127] = True
    y = x.clone()
    y[0, 3, 7], y[0, 20, 1], y[1, 39, 127] = math.inf, math.nan, -math.inf
    cache = fkv.Cache8.zeros(shape, 16)
    fkv.fkv_append_frames_q8(shape, None, None, y.cuda(), y.cuda(), [0], cache)
    want, ws = quantise(torch.where(bad, torch.zeros_like(x), x).float()[:, None], 16)
    for codes, scales in ((cache.K, cache.k_scale), (cache.V, cache.v_scale)):
        assert torch.equal(scales.cpu(), ws)
        c = codes.cpu().reshape(x.shape)
        assert bool(torch.isnan(c.float()[bad]).all())
        assert torch.equal(c.view(torch.uint8)[~bad], want.reshape(x.shape).view(torch.uint8)[~bad])


@pytest.mark.parametrize("halves", [False, True])
def test_append_q8_rotated_not_finite(fkv, halves):
    """A rotated pair with an infinity or a NaN becomes NaN, both channels; everything else as without it."""
    rope = Rope(32, 16, 16, row_tokens=8, halves=halves)
    shape = _shape(fkv, 1, 128, 40, 0, 2, 1)
    x = torch.randn((1, 40, 128), generator=_gen(8)).to(torch.bfloat16)
    y = x.clone()
    hit = torch.zeros(x.shape, dtype=torch.bool)
    for tok, ch, v in ((2, 6, math.inf), (20, 40, math.nan), (39, 63, -math.inf)):
        y[0, tok, ch] = v
        pair = [ch, ch + 64] if halves else [ch & ~1, ch | 1]
        for c in pair:
            x[0, tok, c] = 0                     # (a pair of zeros: no part in the block's scale)
            hit[0, tok, c] = True
            if c != ch:
                y[0, tok, c] = 1
    caches = []
    for t in (x, y):
        caches.append(fkv.Cache8.zeros(shape, 16))
        fkv.fkv_append_frames_q8(shape, rope.make(fkv), [5], t.cuda(), t.cuda(), [1], caches[-1])
    a, b = (c.K.cpu()[:, 1] for c in caches)
    assert torch.equal(caches[0].k_scale, caches[1].k_scale)
    assert torch.equal(a.view(torch.uint8)[~hit], b.view(torch.uint8)[~hit])
    assert bool(torch.isnan(b.float()[hit]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["video", "sequence", "partial"])
@pytest.mark.parametrize("d,F,block", [(128, 70, 32), (64, 129, 128), (128, 1, 16)])
def test_append_q8_rotated(fkv, dtype, name, d, F, block):
    heads, n = 3, 2
    rope = _rope(name, d, F)
    shape = _shape(fkv, heads, d, F, 0, 3, 1, dtype=dtype)
    _, K, V = _projection(_gen(7), n * F, heads, d, dtype)
    pos, slots = [41, 42], [2, 0]
    cache = fkv.Cache8.zeros(shape, block)
    fkv.fkv_append_frames_q8(shape, rope.make(fkv), pos, K, V, slots, cache)
    want = rotate64(K.cpu(), rope, pos, F).reshape(heads, n, F, d)
    slack = rotation_slack(K.cpu(), rope).reshape(want.shape)
    got_s = cache.k_scale.cpu()[:, slots]
    nb = got_s.shape[2]
    for b in range(nb):
        top = want[:, :, b * block:(b + 1) * block].abs().amax((2, 3))
        for i in range(heads):
            for f in range(n):
                k, t, e = math.log2(float(got_s[i, f, b])), float(top[i, f]), float(slack.max())
                assert k in (exponent_of(t - e), exponent_of(t + e))
    got = values(cache.K.cpu(), cache.k_scale.cpu(), block)[:, slots]
    unit = got_s.double().repeat_interleave(block, -1)[:, :, :F, None]
    bound = torch.maximum(half_step(E4M3) * want.abs(), unit * 2.0 ** -10) + 1.07 * slack
    assert bool(((got - want).abs() <= bound).all())
    vq, vs = quantise(V.cpu().float().reshape(heads, n, F, d), block)
    assert torch.equal(cache.v_scale.cpu()[:, slots], vs)
    assert torch.equal(cache.V.cpu().view(torch.uint8)[:, slots], vq.view(torch.uint8))


# -------------------------------------------------------- scoring and attention
def _budgets(n_static, n_dyn, recent, k, scope, sink=1):
    return [W.HeadBudget(W.STATIC, sink, recent)] * n_static + [W.HeadBudget(W.DYNAMIC, sink, 0, k, scope)] * n_dyn


def _cache(fkv, shape, block, seed, spread=1.0):
    """A cache of AR(1) keys and random values, quantised by the library itself (tested above)."""
    g = _gen(seed)
    h, cap, F, d = shape.n_heads, shape.cap_frames, shape.frame_tokens, shape.head_dim
    x = torch.randn((h, cap, F, d), generator=g)
    for t in range(1, cap):
        x[:, t] = 0.9 * x[:, t - 1] + 0.44 * x[:, t]
    x *= torch.exp(spread * torch.randn((h, 1, F, 1), generator=g))
    v = torch.randn((h, cap, F, d), generator=g) * torch.exp(spread * torch.randn((h, cap, F, 1), generator=g))
    cache = fkv.Cache8.zeros(shape, block)
    rows = [t.reshape(h, cap * F, d).to(torch.bfloat16).cuda() for t in (x, v)]
    fkv.fkv_append_frames_q8(shape, None, None, *rows, list(range(cap)), cache)
    return cache


@pytest.mark.parametrize("heads,d,F,H,L,block,k,scope", [
    (3, 128, 128, 5, 64, 64, 1, W.SCOPE_FRAME), (4, 64, 130, 4, 26, 16, 2, W.SCOPE_FRAME),
    (2, 128, 65, 6, 65, 32, 3, W.SCOPE_GLOBAL), (3, 64, 33, 7, 99, 128, 1, W.SCOPE_GLOBAL),
    (2, 64, 1, 9, 1, 16, 4, W.SCOPE_GLOBAL), (2, 128, 1560, 3, 1560, 64, 1, W.SCOPE_GLOBAL),
    (2, 128, 520, 2, 2, 16, 100, W.SCOPE_FRAME)])
def test_score_select_q8(fkv, heads, d, F, H, L, block, k, scope):
    """The cosine in 64 bits, within three roundings of a chain of four products for the product's sum, half as many
    for each norm, and the score's own; the selection of those scores, and that of the bf16 cache of the same values."""
    budgets = _budgets(1, heads - 1, 1, k, scope)
    shape = _shape(fkv, heads, d, F, H, H + 1, 2, L)
    hs = fkv.make_heads(budgets)
    cache = _cache(fkv, shape, block, 11)
    slots = np.random.default_rng(2).permutation(H + 1)[:H].tolist()
    K_cur = torch.randn((heads, 2 * F, d), generator=_gen(12)).to(torch.bfloat16).cuda()
    n_seg = fkv.fkv_num_segments(shape)

    def outputs():
        return (torch.full((heads, n_seg), 9.0, device="cuda"), torch.full((heads, n_seg), 77, dtype=torch.int32, device="cuda"),
                torch.full((heads,), 55, dtype=torch.int32, device="cuda"))
    a, b = outputs(), outputs()
    ws = fkv.fkv_score_select_q8(shape, hs, cache, slots, K_cur, *a)
    fkv.fkv_score_select_q8(shape, hs, cache, slots, K_cur, *a, workspace=ws)      # the workspace serves again
    val = values(cache.K.cpu(), cache.k_scale.cpu(), block)
    plain = val.to(torch.bfloat16)
    assert torch.equal(plain.double(), val)                                      # exact in bf16, as documented
    fkv.fkv_score_select(shape, hs, plain.cuda(), slots, K_cur, *b)
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    c = outputs()
    fkv.fkv_select(shape, hs, a[0], c[1], c[2])
    assert torch.equal(a[1], c[1]) and torch.equal(a[2], c[2])
    assert bool((a[0][0] == 9).all()) and bool((a[1][0] == 77).all()) and int(a[2][0]) == 55     # the static head's rows
    seq = torch.cat([val[:, slots].reshape(heads, H * F, d), K_cur.cpu().double()], 1)
    for g in range(n_seg):
        lo, hi = g * L, min(g * L + L, H * F)
        u, w = seq[1:, lo:hi].flatten(1), seq[1:, lo + F:hi + F].flatten(1)
        c = (u * w).sum(1) / ((u * u).sum(1) * (w * w).sum(1)).sqrt()
        assert bool(((a[0].cpu().double()[1:, g] - c).abs() <= F32_STEP * c.abs() + (3 + 3 * c.abs()) * F32_STEP).all())


def test_score_select_q8_ties_and_ends(fkv):
    """Equal frames score exactly one and go to the lower index; blocks at both ends of the scale's range keep their
    cosine; an all-zero frame scores zero; a NaN code spoils its own segments."""
    heads, d, F, H = 2, 64, 48, 6
    shape = _shape(fkv, heads, d, F, H, H, 1)
    hs = fkv.make_heads(_budgets(0, 2, 0, 3, W.SCOPE_GLOBAL, sink=0))
    g = _gen(13)
    one = torch.randn((heads, 1, F, d), generator=g)
    x = one.expand(-1, H, -1, -1).clone()
    x[1, :, :16] *= 2.0 ** -118
    x[1, :, 16:32] *= 2.0 ** 110
    x[1, 3] = 0
    cache = fkv.Cache8.zeros(shape, 16)
    rows = x.reshape(heads, H * F, d).to(torch.bfloat16).cuda()
    fkv.fkv_append_frames_q8(shape, None, None, rows, rows, list(range(H)), cache)
    cur = torch.randn((heads, F, d), generator=g).to(torch.bfloat16).cuda()
    scores = torch.zeros((heads, H), device="cuda")
    kept, kv = torch.zeros((heads, H), dtype=torch.int32, device="cuda"), torch.zeros(heads, dtype=torch.int32, device="cuda")
    fkv.fkv_score_select_q8(shape, hs, cache, list(range(H)), cur, scores, kept, kv)
    assert scores[0, :5].tolist() == [1.0] * 5 and kept[0].tolist() == [0, 1, 5, -1, -1, -1]
    assert scores[1, :5].tolist() == [1.0, 1.0, 0.0, 0.0, 1.0] and kept[1].tolist()[:3] == [2, 3, 5]
    cache.K.view(torch.uint8)[0, 4, 7, 7] = 0x7f
    fkv.fkv_score_select_q8(shape, hs, cache, list(range(H)), cur, scores, kept, kv)
    assert scores[0].isnan().tolist() == [False, False, False, True, True, False] and kept[0].tolist()[:3] == [0, 1, 5]


def test_score_select_q8_without_history(fkv):
    shape = _shape(fkv, 2, 64, 8, 0, 2, 1)
    hs = fkv.make_heads(_budgets(1, 1, 1, 1, W.SCOPE_GLOBAL))
    cache = fkv.Cache8.zeros(shape, 16)
    kv = torch.full((2,), 5, dtype=torch.int32, device="cuda")
    empty = torch.empty((2, 0), device="cuda")
    fkv.fkv_score_select_q8(shape, hs, cache, [], torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda"), empty,
                            empty.int(), kv)
    assert kv.tolist() == [5, 0]


class Attend:
    """One attention call's inputs, its run and its check against 64 bits."""

    def __init__(self, fkv, heads=3, d=128, F=64, H=4, L=None, block=64, n_q=5, n_cur=3, budgets=None, seed=21, qs=1.0,
                 spread=0.5):
        self.fkv, L = fkv, F if L is None else L
        budgets = _budgets(1, heads - 1, 1, 1, W.SCOPE_GLOBAL) if budgets is None else budgets
        self.budgets, self.shape = budgets, _shape(fkv, heads, d, F, H, H + 2, 1, L)
        self.heads, self.block, self.scale = fkv.make_heads(budgets), block, 1 / math.sqrt(d)
        self.cache = _cache(fkv, self.shape, block, seed, spread)
        g = _gen(seed + 1)
        self.slots = np.random.default_rng(seed).permutation(H + 2)[:H].tolist()
        rnd = lambda n: torch.randn((heads, n, d), generator=g)  # noqa: E731
        self.Q, self.K_cur, self.V_cur = (rnd(n_q) * qs).to(torch.bfloat16), rnd(n_cur).to(torch.bfloat16), rnd(n_cur).to(torch.bfloat16)
        n_seg = fkv.fkv_num_segments(self.shape)
        self.kept = np.full((heads, n_seg), -1, np.int32)
        self.kv_len = np.zeros(heads, np.int32)
        rng = np.random.default_rng(seed + 2)
        for h, b in enumerate(budgets):
            if b.type == W.DYNAMIC and H > 0:
                n = int(rng.integers(0, min(b.keep_k, n_seg) + 1)) if h % 2 else min(b.keep_k, n_seg)
                ids = np.sort(rng.permutation(n_seg)[:n])
                self.kept[h, :n] = ids
                self.kv_len[h] = sum(min(L, H * F - int(g) * L) for g in ids)

    def run(self, workspace="own", lse=True, stream=None, cur=True):
        f = self.fkv
        n_cur = self.K_cur.shape[1] if cur else 0
        O = torch.full_like(self.Q, 5.0).cuda()
        out = torch.full(self.Q.shape[:2], 6.0, device="cuda") if lse else None
        if workspace == "own":
            n = f.fkv_chunk_attention_q8_workspace_size(self.shape, self.heads, self.Q.shape[1], n_cur)
            workspace = torch.zeros(max(n, 1), dtype=torch.uint8, device="cuda")
        dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
        f.fkv_chunk_attention_q8(self.shape, self.heads, self.cache, self.slots, dev(self.kept), dev(self.kv_len), self.Q.cuda(),
                                 self.K_cur.cuda() if cur else None, self.V_cur.cuda() if cur else None, self.scale, O, out,
                                 workspace, stream=stream)
        torch.cuda.synchronize()
        return O, out

    def sources(self, h):
        s = self.shape
        tok = kept_tokens(h, self.budgets, self.kept, self.kv_len, s.hist_frames, s.frame_tokens, s.seg_tokens)
        K = values(self.cache.K.cpu(), self.cache.k_scale.cpu(), self.block)[h][self.slots].reshape(-1, s.head_dim)[tok]
        V = values(self.cache.V.cpu(), self.cache.v_scale.cpu(), self.block)[h][self.slots].reshape(-1, s.head_dim)[tok]
        return K, V

    def check(self, O, lse, cur=True):
        O, lse = O.cpu().double(), None if lse is None else lse.cpu().double()
        for h in range(self.shape.n_heads):
            K, V = self.sources(h)
            if cur:
                K, V = torch.cat([K, self.K_cur[h].double()]), torch.cat([V, self.V_cur[h].double()])
            want, bound, wl, bl = attention_bounds(self.Q[h].double(), K, V, self.scale)
            err = (O[h] - want).abs()
            assert bool((err <= bound).all()), (h, float((err / bound).max()))
            if lse is not None:
                same = torch.isinf(wl) & (lse[h] == wl)
                assert bool((same | ((lse[h] - wl).abs() <= bl)).all()), (h, float((lse[h] - wl).abs().max()))


SIZES = [
    dict(heads=3, d=128, F=64, H=4, n_q=1, n_cur=1),                                  # one query token
    dict(heads=2, d=64, F=64, H=4, n_q=1, n_cur=0),
    dict(heads=4, d=128, F=1, H=7, n_q=3, n_cur=2, block=16),                         # frames of one token
    dict(heads=3, d=64, F=5, H=9, n_q=17, n_cur=1, block=16),                         # a page ends inside a tile, often
    dict(heads=3, d=128, F=100, H=5, L=25, n_q=16, n_cur=33, block=32,
         budgets=_budgets(1, 2, 2, 9, W.SCOPE_GLOBAL)),                               # segments inside blocks
    dict(heads=3, d=128, F=33, H=8, L=99, n_q=2, n_cur=64, block=128,
         budgets=_budgets(1, 2, 3, 3, W.SCOPE_GLOBAL)),                               # segments of frames, the last short
    dict(heads=2, d=64, F=333, H=13, L=111, n_q=131, n_cur=131, block=32,
         budgets=_budgets(1, 1, 3, 30, W.SCOPE_GLOBAL)),
    dict(heads=2, d=128, F=390, H=6, n_q=40, n_cur=390, budgets=_budgets(1, 1, 4, 5, W.SCOPE_GLOBAL)),
    dict(heads=1, d=128, F=1560, H=10, n_q=1, n_cur=0, budgets=_budgets(1, 0, 10, 0, W.SCOPE_GLOBAL)),   # many parts
    dict(heads=5, d=64, F=16, H=3, n_q=300, n_cur=300, block=16),
    dict(heads=2, d=128, F=65, H=0, n_q=9, n_cur=70),                                 # nothing cached
    dict(heads=16, d=64, F=60, H=12, n_q=650, n_cur=5, budgets=_budgets(8, 8, 11, 9, W.SCOPE_GLOBAL)),   # 48-row tiles
    dict(heads=16, d=64, F=60, H=12, n_q=500, n_cur=130, budgets=_budgets(8, 8, 11, 9, W.SCOPE_GLOBAL)),  # 32-row tiles
    dict(heads=12, d=128, F=1300, H=5, n_q=81, n_cur=81, budgets=_budgets(6, 6, 5, 5, W.SCOPE_GLOBAL)),  # 32-row, in parts
]


@pytest.mark.parametrize("size", [
    dict(heads=9, d=128, F=1560, H=8, n_q=1100, n_cur=1100, budgets=_budgets(5, 4, 8, 8, W.SCOPE_GLOBAL)),
    dict(heads=10, d=64, F=1500, L=500, H=9, n_q=1030, n_cur=37, budgets=_budgets(4, 6, 9, 20, W.SCOPE_GLOBAL))],
    ids=["chunk", "few-current"])
def test_attention_expanded(fkv, size):
    """Large chunks, attended over the expanded copy; the same workspace then serves a small call."""
    a = Attend(fkv, **size)
    n = fkv.fkv_chunk_attention_q8_workspace_size(a.shape, a.heads, a.Q.shape[1], a.K_cur.shape[1])
    copy = 2 * size["heads"] * 2 * size["d"] * size["F"] * size["H"]
    assert n >= copy                                  # it holds the copy: this call takes that way
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")     # no initialisation needed
    O, lse = a.run(ws)
    a.check(O, lse)
    P, _ = a.run(ws, lse=False)
    assert torch.equal(O, P)
    b = Attend(fkv, heads=2, d=128, F=1560, H=10, n_q=3, n_cur=0, budgets=_budgets(2, 0, 10, 0, W.SCOPE_GLOBAL))
    b.check(*b.run(ws))
    assert all(torch.equal(x, y) for x, y in zip(a.run(ws), (O, lse)))


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "-".join(f"{k}{v}" for k, v in s.items() if k != "budgets"))
def test_attention(fkv, size):
    a = Attend(fkv, **size)
    O, lse = a.run()
    a.check(O, lse)
    again, _ = a.run(lse=False)                       # without lse: the same bits
    assert torch.equal(O, again)
    P, pl = a.run(workspace=None)                     # one workgroup per query tile
    a.check(P, pl)


def test_attention_without_keys(fkv):
    """Heads that keep nothing, next to one that does, and no current tokens: zeros and -inf."""
    budgets = [W.HeadBudget(W.STATIC, 0, 0), W.HeadBudget(W.DYNAMIC, 0, 0, 0), W.HeadBudget(W.STATIC, 1, 0)]
    a = Attend(fkv, heads=3, F=70, H=3, n_q=18, budgets=budgets)
    for ws in ("own", None):
        O, lse = a.run(cur=False, workspace=ws)
        assert bool((O[:2] == 0).all()) and bool((lse[:2] == -math.inf).all())
        a.check(O, lse, cur=False)


@pytest.mark.parametrize("qs", [30.0, 300.0])
def test_attention_far_scores(fkv, qs):
    """Scores far apart: all weight on a few keys, maxima that move from tile to tile."""
    a = Attend(fkv, heads=2, d=128, F=200, H=5, n_q=20, n_cur=10, qs=qs, budgets=_budgets(1, 1, 3, 4, W.SCOPE_GLOBAL))
    O, lse = a.run()
    a.check(O, lse)


def test_attention_reads_only_what_is_kept(fkv):
    """NaN in every code and scale that no head keeps (other slots, other frames, rows behind kv_len) changes nothing."""
    a = Attend(fkv, heads=3, d=64, F=50, H=6, L=25, n_q=20, n_cur=7, block=16, budgets=_budgets(1, 2, 2, 5, W.SCOPE_GLOBAL))
    O, lse = a.run()
    keep = torch.zeros((3, 8, 50), dtype=torch.bool)
    for h in range(3):
        for x in kept_tokens(h, a.budgets, a.kept, a.kv_len, 6, 50, 25):
            keep[h, a.slots[int(x) // 50], int(x) % 50] = True
    for t in (a.cache.K, a.cache.V):
        t.view(torch.uint8)[~keep.cuda()] = 0x7f
    used = torch.nn.functional.pad(keep, (0, 14)).reshape(3, 8, 4, 16).any(-1).cuda()
    for s in (a.cache.k_scale, a.cache.v_scale):
        s[~used] = math.nan
    P, pl = a.run()
    assert torch.equal(O, P) and torch.equal(lse, pl)
    a.check(P, pl)


def test_attention_not_finite(fkv):
    """A NaN code, an infinite current key or value reach the rows that the formula says, and no other head."""
    a = Attend(fkv, heads=3, d=64, F=40, H=3, n_q=18, n_cur=9, budgets=_budgets(3, 0, 2, 0, W.SCOPE_GLOBAL))
    clean, _ = a.run()
    a.cache.V.view(torch.uint8)[0, a.slots[2], 11, 5] = 0x7f          # head 0: one value channel of a kept token
    a.K_cur[1, 4, :] = math.inf                                       # head 1: scores of +-inf or NaN
    O, lse = a.run()
    assert torch.equal(O[2], clean[2])
    assert bool(torch.isnan(O[0, :, 5]).all())
    rest = [c for c in range(64) if c != 5]
    assert torch.equal(O[0][:, rest], clean[0][:, rest])
    z = (a.Q[1].double() @ a.K_cur[1].double().T)[:, 4]
    down = z == -math.inf                                             # exp(-inf) = 0: the row is as without the key
    assert bool(torch.isnan(O[1].float()).all(1)[~down.cuda()].all())
    assert bool(torch.isfinite(O[1].float()).all(1)[down.cuda()].all())


def test_attention_bad_lists_stay_inside(fkv):
    """kv_len beyond the history and segment ids out of range are clamped: the call reads the cache only, and other
    heads are right.  (The clamps themselves are host-checked in test_cache8_pages.)"""
    a = Attend(fkv, heads=3, d=64, F=40, H=3, n_q=4, n_cur=2, budgets=_budgets(1, 2, 2, 2, W.SCOPE_GLOBAL))
    good, _ = a.run()
    kept, kv = a.kept.copy(), a.kv_len.copy()
    a.kept[1], a.kv_len[1] = [5000, -7, 2 ** 31 - 1], 2 ** 31 - 1
    O, _ = a.run()
    assert torch.equal(O[0], good[0]) and torch.equal(O[2], good[2])
    a.kept, a.kv_len = kept, kv
    a.kv_len[1] = -3                                                   # below zero: nothing kept
    O, lse = a.run()
    a.kv_len[1], a.kept[1] = 0, -1
    a.check(O, lse)


def test_attention_expanded_bad_lists_stay_inside(fkv):
    """The same of a large chunk: the expanded copy has room for every token that kv_len may claim (the whole history,
    beyond the budgets), and the heads beside the lying one are right."""
    a = Attend(fkv, heads=10, d=64, F=700, H=12, n_q=1600, n_cur=1600, budgets=_budgets(9, 1, 11, 1, W.SCOPE_GLOBAL))
    n = fkv.fkv_chunk_attention_q8_workspace_size(a.shape, a.heads, 1600, 1600)
    assert n >= 2 * 2 * 64 * 10 * 12 * 700
    ws = torch.zeros(n + (1 << 16), dtype=torch.uint8, device="cuda")
    a.kept[9], a.kv_len[9] = np.arange(12), 12 * 700                  # more than its budget keeps: attended as it says
    O, lse = a.run(ws[:n])
    a.check(O, lse)
    a.kept[9], a.kv_len[9] = 2 ** 31 - 1, 2 ** 31 - 1
    O, lse = a.run(ws[:n])
    a.kept[9], a.kv_len[9] = 11, 12 * 700                             # clamped: the last segment over and over
    a.check(O, lse)     # (to the bounds: the parts are cut by every head's length, so other heads' last bits move too)
    assert not bool(ws[n:].any())


def test_attention_repeats_and_shares_a_workspace(fkv):
    """The same bits on every run; one workspace serves calls of other sizes in turn."""
    a = Attend(fkv, heads=2, d=128, F=300, H=6, n_q=3, n_cur=3, budgets=_budgets(1, 1, 5, 5, W.SCOPE_GLOBAL))
    b = Attend(fkv, heads=4, d=64, F=90, H=4, n_q=33, n_cur=0, budgets=_budgets(2, 2, 3, 3, W.SCOPE_GLOBAL))
    size = lambda x: fkv.fkv_chunk_attention_q8_workspace_size(x.shape, x.heads, x.Q.shape[1], x.K_cur.shape[1])  # noqa: E731
    ws = torch.zeros(max(size(a), size(b)), dtype=torch.uint8, device="cuda")
    first, second = a.run(ws), b.run(ws)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(a.run(ws), first))
        assert all(torch.equal(x, y) for x, y in zip(b.run(ws), second))
    a.check(*first)
    b.check(*second)


def test_streams_and_graphs(fkv):
    """A whole turn -- rotate, append, score and select, attend -- on another stream, and captured and replayed with
    new inputs, against the eager result each time."""
    heads, d, F, H, C = 4, 64, 48, 5, 1
    budgets = _budgets(2, 2, 2, 2, W.SCOPE_GLOBAL)
    shape = _shape(fkv, heads, d, F, H, H + 1, C)
    hs, rope = fkv.make_heads(budgets), Rope(12, 10, 10, row_tokens=8).make(fkv)
    cache = _cache(fkv, shape, 16, 31)
    g = _gen(32)
    x = torch.randn((C * F, 3, heads, d), generator=g).to(torch.bfloat16).cuda()
    Q, K, V = (x[:, i].transpose(0, 1) for i in range(3))
    buf = [torch.zeros((heads, C * F, d), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    n_seg = fkv.fkv_num_segments(shape)
    scores = torch.zeros((heads, n_seg), device="cuda")
    kept = torch.full((heads, n_seg), -1, dtype=torch.int32, device="cuda")
    kv = torch.zeros(heads, dtype=torch.int32, device="cuda")
    lse = torch.zeros((heads, C * F), device="cuda")
    ws = torch.zeros(fkv.fkv_score_workspace_size(shape, hs), dtype=torch.uint8, device="cuda")
    wa = torch.zeros(max(1, fkv.fkv_chunk_attention_q8_workspace_size(shape, hs, C * F, C * F)), dtype=torch.uint8, device="cuda")

    def turn(stream=None):
        fkv.fkv_rotate_chunk(shape, rope, [9], Q, K, V, *buf[:3], stream=stream)
        fkv.fkv_append_frames_q8(shape, rope, [9], K, V, [5], cache, stream=stream)
        fkv.fkv_score_select_q8(shape, hs, cache, [0, 1, 2, 3, 4], buf[1], scores, kept, kv, ws, stream=stream)
        fkv.fkv_chunk_attention_q8(shape, hs, cache, [0, 5, 2, 3, 4], kept, kv, buf[0], buf[1], buf[2], 0.125, buf[3], lse,
                                   wa, stream=stream)

    def result():
        torch.cuda.synchronize()
        return [t.clone() for t in (*buf, scores, kept, kv, lse, cache.K.view(torch.uint8), cache.k_scale)]
    turn()
    want = result()
    side = torch.cuda.Stream()
    for t in buf:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    turn(stream=side)
    assert all(torch.equal(a, b) for a, b in zip(result(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn()
    for seed in range(3):
        x.copy_(torch.randn(x.shape, generator=_gen(40 + seed)).to(torch.bfloat16))
        graph.replay()
        got = result()
        turn()
        assert all(torch.equal(a, b) for a, b in zip(result(), got))
