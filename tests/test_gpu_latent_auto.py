"""Latent attention that chooses its form: a batch whose token count is not known has no room for expanded keys and
is served whole all the same."""
import math

import pytest
import torch

from tests.paged_ref import ROT, attend_latent, rel2
from tests.test_gpu_paged_batch import BF, latent_case, view

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("causal,span", [(True, None), (False, None), (True, (0, 50))])
@pytest.mark.parametrize("d,R,seqs", [(64, 256, [(900, 200)]), (128, 512, [(400, 1), (700, 64), (130, 130)])])
def test_unknown_token_count(fkv, causal, span, d, R, seqs):
    heads = 3
    x, Q, W_k, W_v = latent_case(seqs, 48, heads, d, R, 90)
    b = x.batch(fkv, sum_len=0)
    O = view(torch.full((heads, x.n_tokens, d), 7.0, dtype=BF), "token")
    fkv.fkv_latent_attention(b, view(Q, "token"), x.K.cuda(), W_k.cuda(), W_v.cuda(), 1 / math.sqrt(d + ROT), O, causal=causal, span=span)
    O = O.cpu()
    ref, _ = attend_latent(x, Q, W_k, W_v, 1 / math.sqrt(d + ROT), causal, span)
    a, e = x.starts[0], x.starts[-1]
    # absorbed queries and the output: two roundings of at most half a step of bf16, 2^-8 / sqrt 3 each
    assert rel2(O[:, a:e], ref[:, a:e]) <= 2.0 ** -8
    assert bool((O[:, :a] == 7).all()) and bool((O[:, e:] == 7).all())
