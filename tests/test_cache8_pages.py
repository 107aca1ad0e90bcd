"""Where a kept token lies (the 8-bit attention's lookup), modelled on the host:
whatever kept_seg and kv_len hold, the row stays inside the head's cache, and
for lists that agree it is the token's own row."""
import numpy as np
import pytest


def magic(P):
    return 0 if P <= 1 else (1 << 64) // P + 1


def div(j, m):
    """j / P by multiplication, as the kernel computes it: 32-bit words, the low word's high half only."""
    if m == 0:
        return j
    hi, lo = m >> 32, m & 0xffffffff
    return (j * hi + ((j * lo) >> 32)) >> 32


def place(j, F, L, H, n_seg, segs, slots):
    q = div(j, magic(L))
    assert 0 <= q < n_seg
    g = min(max(int(segs[q]), 0), n_seg - 1)
    tok = min(g * L + (j - q * L), H * F - 1)
    assert tok < 2 ** 31
    t = div(tok, magic(F))
    return slots[t] * F + tok - t * F


@pytest.mark.parametrize("P", [1, 2, 3, 5, 7, 25, 64, 111, 333, 1560, 8160, 65537, (1 << 24) - 1, 1 << 24, (1 << 30) + 1])
def test_division_by_multiplication(P):
    rng = np.random.default_rng(P)
    top = (1 << 31) - 1
    js = {0, 1, P - 1, P, P + 1, top, top - 1, (top // P) * P, max(0, (top // P) * P - 1)}
    js |= {int(k) * P + e for k in rng.integers(0, top // P + 1, 2000) for e in (-1, 0, 1)}
    js |= {int(v) for v in rng.integers(0, top, 2000)}
    for j in js:
        if 0 <= j <= top:
            assert div(j, magic(P)) == j // P


@pytest.mark.parametrize("F,L,H,cap", [(1, 1, 7, 9), (5, 1, 9, 9), (100, 25, 5, 6), (33, 99, 8, 10), (64, 64, 4, 4), (10, 40, 3, 5)])
def test_rows_stay_inside(F, L, H, cap):
    n_seg = -(-H * F // L)
    rng = np.random.default_rng(F * L)
    slots = rng.permutation(cap)[:H]
    wild = rng.integers(-2 ** 31, 2 ** 31, n_seg)
    for j in range(H * F):                            # (kv_len is clamped to H*F before)
        assert 0 <= place(j, F, L, H, n_seg, wild, slots) < cap * F
    for trial in range(20):
        ids = np.sort(rng.permutation(n_seg)[:int(rng.integers(1, n_seg + 1))])
        tokens = [x for g in ids for x in range(g * L, min(g * L + L, H * F))]
        segs = np.full(n_seg, -1)
        segs[:len(ids)] = ids
        for j, x in enumerate(tokens):
            assert place(j, F, L, H, n_seg, segs, slots) == slots[x // F] * F + x % F
