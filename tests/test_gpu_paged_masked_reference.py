"""Attention whose first tile of keys holds, beside the first that a row sees, hidden ones with far larger scores."""
import math

import pytest
import torch

from tests.paged_ref import Paged, attend
from tests.test_gpu_paged_batch import BF, run_attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("high,low", [(-117.0, -126.5), (-116.5, -126.5), (-99.0, -126.5), (-60.0, -90.0), (-125.0, -127.0)])
@pytest.mark.parametrize("new", [1, 3, 70])
def test_hidden_keys_far_above(fkv, new, high, low, workspace):
    """2^18 visible keys, scores of two sizes in turn, in log2 units below the hidden ones' (a key's first channel is its
    score): the smaller ones' weights have to be there, too."""
    d, recent, hidden = 64, 1 << 18, 63                    # (the first tile a row sees begins with hidden keys)
    x = Paged([(hidden + recent + new, new)], 1024, 1, d, seed=90)
    x.K.zero_()
    t = torch.arange(x.seqs[0][0])
    score = torch.where(t < hidden, 0.0, torch.where(t % 2 == 1, high, low)).to(BF)
    x.K[x.table[0].long()[t // 1024], 0, t % 1024, 0] = score
    Q = torch.zeros((1, x.n_tokens, d), dtype=BF)
    Q[..., 0] = 1.0
    spans = [(0, recent)]
    O, lse = run_attend(fkv, x, Q, causal=False, spans=spans, workspace=workspace, sum_len=0, scale=math.log(2.0))
    ref, rl, A, top = attend(x, Q, math.log(2.0), False, spans)
    # Scores are single products.  scale log2 e is off by three roundings, the exponent by one more, of 127 log2 units:
    # 4 * 127 * 2^-24; the exponentials by 2^-21; the log by its own rounding, of 100.  A thread sums four keys of a tile of 32 and
    # adds them to its sum, 2^13 + 3 times, or (more than 64 rows) 16 keys of a tile of 64 one by one, 2^16 + 16 times.
    adds = (1 << 13) + 3 if new <= 64 else (1 << 16) + 16
    tol = math.log(2.0) * 4 * 127 * 2.0 ** -24 + 2.0 ** -21 + 100 * 2.0 ** -24 + (adds + 8) * 2.0 ** -24
    assert float((lse.double() - rl).abs().max()) <= tol
    # half a step of bf16 each for probabilities and output
    assert bool(((O.double() - ref).abs() <= 2.0 ** -7 * (A + ref.abs()) + 1e-30).all())
