"""Outputs are divided by the sum of the weights as they weigh the values, rounded: a row that sees one key has its
value, bit for bit, whatever hidden keys its reference comes from, and asking for lse changes nothing."""
import math

import pytest
import torch

from tests.paged_ref import Paged, attend, close_lse
from tests.test_gpu_paged_batch import BF, run_attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


FEW = [(812, 1), (93, 5), (1, 1), (300, 16), (64, 64), (33, 20)]
MANY = [(300, 300), (1000, 129), (97, 97), (129, 1), (700, 530)]


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("d,heads,kv,seqs,sum_len", [
    (64, 4, 4, FEW, None), (128, 6, 2, FEW, None), (64, 4, 4, MANY, 0), (128, 4, 2, MANY, 0), (128, 2, 2, [(600, 530)], 0)])
def test_one_key_a_row(fkv, d, heads, kv, seqs, sum_len, workspace):
    """Each token sees itself alone, and the first tile of keys is full of hidden ones."""
    x = Paged(seqs, 16, kv, d, seed=110)
    Q = x.rows(heads, d)
    spans = [(0, 0)] * kv
    O, lse = run_attend(fkv, x, Q, spans=spans, sum_len=sum_len, workspace=workspace)
    for i, (length, new) in enumerate(seqs):
        for h in range(heads):
            v = x.of(x.V, i, h * kv // heads)[length - new:]
            # p v and p are exact in fp32, and v (1 + 2^-23) rounds to v
            assert torch.equal(O[h, x.starts[i]:x.starts[i + 1]], v), (i, h)
    _, rl, _, top = attend(x, Q, 1 / math.sqrt(d), True, spans)
    assert close_lse(lse, rl, top, d, 1)
    without, _ = run_attend(fkv, x, Q, spans=spans, sum_len=sum_len, workspace=workspace, lse=False)
    assert torch.equal(O, without)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("d,heads,kv,seqs,sum_len", [
    (64, 4, 4, FEW, None), (128, 6, 2, FEW, None), (64, 4, 4, MANY, 0), (128, 4, 2, MANY, 0)])
def test_lse_changes_nothing(fkv, d, heads, kv, seqs, sum_len, workspace, causal):
    x = Paged(seqs, 16, kv, d, seed=111)
    Q = x.rows(heads, d)
    outs = [run_attend(fkv, x, Q, causal=causal, sum_len=sum_len, workspace=workspace, lse=lse)[0] for lse in (True, False)]
    assert torch.equal(*outs)
