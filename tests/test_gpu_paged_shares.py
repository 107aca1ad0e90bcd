"""The launch for many rows with many items to a workgroup, whole ones and cut ones in turn, every output against 64 bits;
latent attention row by row."""
import math

import pytest
import torch

from tests.paged_ref import ROT, Paged, mask, weighted
from tests.test_gpu_paged_batch import BF, check, latent_case, run_attend, run_latent

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


# 16 key heads, 2 or 3 row tiles a sequence and head, 24 sequences: some 1000 items for 256 workgroups (256 rows a tile), or 512 (128)
LONG = [(520 + 7 * (i % 5), 520 + 3 * (i % 4)) if i % 3 else (900, 530) for i in range(24)]
SHORT = [(300 + i, 270 + i) for i in range(28)]
MIXED = [(560, 560)] + [(70 + i, 65) for i in range(60)] + [(1, 1), (900, 3), (0, 0)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lse", [True, False])
@pytest.mark.parametrize("d,heads,kv,seqs,spans", [
    (64, 16, 16, LONG, None), (128, 16, 16, SHORT, None), (64, 16, 16, SHORT, None), (64, 16, 8, MIXED, None),
    (128, 16, 16, MIXED, None), (64, 16, 16, LONG, [(0, 0), (33, 100), (0, -1), (700, 5)] * 4)])
def test_many_items_to_a_workgroup(fkv, d, heads, kv, seqs, spans, lse, causal):
    x = Paged(seqs, 48, kv, d, seed=100, spare=1, before=2)
    Q = x.rows(heads, d)
    O, log = run_attend(fkv, x, Q, causal=causal, spans=spans, lse=lse, sum_len=0)
    if lse:
        check(x, Q, O, log, causal, spans)
        return
    # Without lse the sum is of the rounded weights: another half step of bf16 on the normaliser.
    a, e = x.starts[0], x.starts[-1]
    rows = by_rows(x, Q, lambda i, h: (x.of(x.K, i, h * kv // heads).double(), x.of(x.V, i, h * kv // heads).double()),
                   1 / math.sqrt(d), causal, lambda h: spans and spans[h * kv // heads])
    # weights, normaliser and output: half a step each of the sum of the weighted values; scores and sums in fp32
    for i, h, ref, A, top in rows:
        out = O[h, x.starts[i]:x.starts[i + 1]].double()
        tol = 3 * 2.0 ** -8 * (A + ref.abs()) + (torch.expm1(4 * (d + 2) * 2.0 ** -24 * top) + 2.0 ** -16)[:, None] * A
        assert bool(((out - ref).abs() <= tol + 1e-30).all()), (i, h)
    assert bool((O[:, :a] == 7).all()) and bool((O[:, e:] == 7).all())


def by_rows(x, Q, keys, scale, causal, span):
    """(sequence, head, outputs, sums of p |v|, largest sum of |q| |k| of a row) of every sequence and head."""
    for i, (length, new) in enumerate(x.seqs):
        if not new:
            continue
        for h in range(Q.shape[0]):
            k, v = keys(i, h)
            q = Q[h, x.starts[i]:x.starts[i + 1]].double()
            seen = mask(length, new, causal, span(h))
            o, _, A = weighted(q @ k.T * scale, seen, v)
            top = torch.where(seen, q.abs() @ k.abs().T * scale, 0.0).amax(1) if length else torch.zeros(new, dtype=torch.float64)
            yield i, h, o, A, top


@pytest.mark.parametrize("form", ["absorbed", "expanded", "auto"])
@pytest.mark.parametrize("d,R,heads,seqs", [
    (64, 256, 16, [(300 + i, 270 + i) for i in range(20)]), (128, 512, 5, [(700, 1), (300, 300), (64, 64), (90, 63), (1, 1), (450, 70)])])
def test_latent_row_by_row(fkv, form, d, R, heads, seqs):
    """Every element of every token and head."""
    x, Q, W_k, W_v = latent_case(seqs, 48, heads, d, R, 101)
    O = run_latent(fkv, x, Q, W_k, W_v, form=form)
    scale, half = 1 / math.sqrt(d + ROT), 2.0 ** -8
    for i, (length, new) in enumerate(seqs):
        row = x.of(x.K, i, 0).double()
        c, r = row[:, :R], row[:, R:]
        seen = mask(length, new, True, None)
        for h in range(heads):
            wk, wv = W_k[h].double(), W_v[h].double()
            q = Q[h, x.starts[i]:x.starts[i + 1]].double()
            qc, qr = q[:, :d], q[:, d:]
            k, v = c @ wk.T, c @ wv.T
            ref, _, A = weighted((qc @ k.T + qr @ r.T) * scale, seen, v)
            # A score's own error: half a step of bf16 of each absorbed query channel, or of each expanded key channel, and
            # R + d + 66 roundings in fp32 of the absolute sums.
            full = qc.abs() @ wk.abs() @ c.abs().T + qr.abs() @ r.abs().T
            err = scale * (half * torch.maximum((qc @ wk).abs() @ c.abs().T, qc.abs() @ k.abs().T) + (R + d + 66) * 2.0 ** -24 * full)
            err = torch.where(seen, err, 0.0).amax(1, keepdim=True)
            # It moves weights and normaliser; then half a step each of weights, normaliser, values and the output, and the
            # sums over keys and latent channels in fp32, of the absolute products.
            _, _, V = weighted((qc @ k.T + qr @ r.T) * scale, seen, c.abs() @ wv.abs().T)
            tol = torch.expm1(2 * err) * A + 3 * half * (1 + 2 * half) * A + half * ref.abs() + (R + length + 16) * 2.0 ** -24 * V + 2.0 ** -20 * A
            out = O[h, x.starts[i]:x.starts[i + 1]].double()
            assert bool(((out - ref).abs() <= tol + 1e-30).all()), (i, h)
