"""Plain forms in 64 bits of the position rotation, the 8-bit rolling cache and
the attention over it, for the tests (numpy and torch on the CPU; no code of the
library)."""
from __future__ import annotations

import math

import numpy as np
import torch

E4M3 = torch.float8_e4m3fn
F32_STEP = 2.0 ** -24          # half a step of fp32, relative


def half_step(dtype) -> float:
    """Largest relative error of one rounding to ``dtype``."""
    return torch.finfo(dtype).eps / 2


class Rope:
    def __init__(self, frame_pairs, row_pairs=0, col_pairs=0, row_tokens=1, token_step=0, theta=10000.0, halves=False):
        self.counts = (frame_pairs, row_pairs, col_pairs)
        self.row_tokens, self.token_step, self.theta, self.halves = row_tokens, token_step, theta, halves

    def make(self, fkv):
        return fkv.make_rope(*self.counts, row_tokens=self.row_tokens, token_step=self.token_step, theta=self.theta,
                             pairing=fkv.FKV_PAIR_HALVES if self.halves else fkv.FKV_PAIR_ADJACENT)


def pairs(x: torch.Tensor, halves: bool):
    """The two channels of every pair of x [..., d]."""
    if halves:
        return x[..., :x.shape[-1] // 2], x[..., x.shape[-1] // 2:]
    return x[..., 0::2], x[..., 1::2]


def rotate64(x: torch.Tensor, rope: Rope, frame_pos, F: int) -> torch.Tensor:
    """x [heads][n*F][d] rotated, in 64 bits."""
    x = x.double()
    d = x.shape[-1]
    p = np.arange(F)
    ang = np.zeros((len(frame_pos), F, d // 2))
    for f, t in enumerate(frame_pos):
        where = (t + rope.token_step * p, p // rope.row_tokens, p % rope.row_tokens)
        j = 0
        for n, pos in zip(rope.counts, where):
            for i in range(n):
                ang[f, :, j] = pos * rope.theta ** (-i / n)
                j += 1
    ang = torch.from_numpy(ang.reshape(-1, d // 2))
    a, b = pairs(x, rope.halves)
    u, v = a * torch.cos(ang) - b * torch.sin(ang), a * torch.sin(ang) + b * torch.cos(ang)
    return torch.cat([u, v], -1) if rope.halves else torch.stack([u, v], -1).flatten(-2)


def rotation_slack(x: torch.Tensor, rope: Rope) -> torch.Tensor:
    """Bound on what fp32 arithmetic moves a rotated element by, beside its last
    rounding: sine and cosine are off by at most 2^-23 (the angle's remainder kept to
    2^-24 of its size and below 1, and a step of their own), the two products and
    their sum by three half steps: below 2^-21 of |x| + |y|."""
    a, b = pairs(x.double().abs(), rope.halves)
    s = (a + b) * 2.0 ** -21
    return torch.cat([s, s], -1) if rope.halves else torch.stack([s, s], -1).flatten(-2)


def exponent_of(amax: float) -> int:
    """k of the block's scale 2^k, by the definition."""
    if amax == 0:
        return 0
    k = -100
    while k < 119 and amax > 448.0 * 2.0 ** k:
        k += 1
    return k


def quantise(x: torch.Tensor, block: int):
    """Codes (float8) and scales of x [heads][frames][F][d] (fp32 values): the
    definition, block by block."""
    h, n, F, d = x.shape
    nb = -(-F // block)
    scales = torch.empty((h, n, nb))
    codes = torch.empty((h, n, F, d), dtype=E4M3)
    for b in range(nb):
        part = x[:, :, b * block:(b + 1) * block].double()
        mag = torch.where(torch.isfinite(part), part.abs(), torch.zeros_like(part)).amax((2, 3))
        for i in range(h):
            for f in range(n):
                scales[i, f, b] = 2.0 ** exponent_of(float(mag[i, f]))
        y = part / scales[:, :, b, None, None].double()
        y = torch.where(torch.isfinite(part), y.clamp(-448, 448), torch.full_like(y, math.nan))
        codes[:, :, b * block:(b + 1) * block] = y.float().to(E4M3)   # (exact in fp32: a power of two divides)
    return codes, scales


def values(codes: torch.Tensor, scales: torch.Tensor, block: int) -> torch.Tensor:
    """What the codes stand for, fp64 [heads][cap][F][d]."""
    F = codes.shape[2]
    return codes.double() * scales.double().repeat_interleave(block, -1)[:, :, :F, None]


def kept_tokens(h, heads, kept_seg, kv_len, H, F, L):
    """Logical history tokens that head h attends, in order."""
    b = heads[h]
    if b.type == 0:
        t = [t for t in range(H) if t < b.sink_frames or t >= H - b.recent_frames]
        return np.array([x for f in t for x in range(f * F, f * F + F)], np.int64)
    out = []
    for g in kept_seg[h]:
        if g >= 0:
            out += list(range(int(g) * L, min(int(g) * L + L, H * F)))
    return np.array(out, np.int64)[:int(kv_len[h])]


def attend64(q, K, V, scale):
    """O, lse, the mean |v| under the same weights and the bound of the score's
    fp32 accumulation, for q [n][d], K, V [m][d] in 64 bits."""
    if K.shape[0] == 0:
        n, d = q.shape
        return torch.zeros(n, d).double(), torch.full((n,), -math.inf).double(), torch.zeros(n, d).double(), torch.zeros(n)
    z = scale * (q @ K.T)
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    size = scale * (q.abs() @ K.abs().T).amax(1)
    return p @ V, lse, p @ V.abs(), size


def attention_bounds(q, K, V, scale):
    """(O, its bound, lse, its bound): probabilities rounded to bf16 (half a step
    each, on the weighted |v|), the output rounded once, products and sums in
    fp32 (the score's d products, the sum over m keys, exp2 to two steps)."""
    O, lse, mass, size = attend64(q, K, V, scale)
    m, d = max(K.shape[0], 1), q.shape[1]
    dz = size * (d + 4) * F32_STEP + 2.0 ** -21 * (1 + lse.abs().nan_to_num(0, 0, 0)).clamp(min=1)
    rel = half_step(torch.bfloat16) + 2 * dz + (m + 64) * 2 * F32_STEP
    return (O, rel[:, None] * mass * 1.01 + half_step(torch.bfloat16) * O.abs() * 1.01 + 1e-30, lse,
            dz + (m + 64) * F32_STEP + 4 * F32_STEP * lse.abs().nan_to_num(0, 0, 0))
