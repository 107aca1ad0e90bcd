"""Paged batches whose starts fall: each start is held to the largest before it, so every row belongs to one sequence
at most.  Outputs, log sums and pages against 64 bits over the batch that is left, with guards around what is written."""
import math
import random

import pytest
import torch

from tests.paged_ref import ROT, Paged, attend, attend_latent, close, close_lse, rel2
from tests.test_gpu_paged_batch import BF, latent_case

pytestmark = pytest.mark.gpu
GUARD, FILL = 4096, 7.0


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


def wandering(n, seed):
    rng = random.Random(seed)
    return [max(i // 2 + rng.randint(-4, 4), 0) for i in range(n + 1)]


CASES = [
    ([300, 400, 5000, 70, 600], [0, 10, 5, 30, 20, 50], 52),
    ([40] * 130, wandering(130, 1), 66),
    ([200 + i for i in range(20)], [5, 95, 0, 90] * 5 + [100], 110),
    ([80] * 1023 + [30000], [0, 64] * 512 + [0], 64),            # every second sequence claims every row
]


def held(starts, n_tokens):
    out, at = [], 0
    for s in starts:
        at = max(at, min(max(s, 0), n_tokens))
        out.append(at)
    return out


def batch(fkv, x, lens, starts, n_tokens, **kw):
    """The batch as it is given, and x as it is held."""
    x.n_tokens = n_tokens
    x.seqs, x.starts = [(n, 0) for n in lens], starts
    b = x.batch(fkv, max_new=n_tokens, **kw)
    x.starts = held(starts, n_tokens)
    x.seqs = [(n, x.starts[i + 1] - x.starts[i]) for i, n in enumerate(lens)]
    return b


def guarded(shape, dtype):
    """A filled tensor between guards, and the whole."""
    n = math.prod(shape)
    whole = torch.full((n + 2 * GUARD,), FILL, dtype=dtype, device="cuda")
    return whole[GUARD:GUARD + n].view(shape), whole


def untouched(whole):
    return bool((whole[:GUARD] == FILL).all()) and bool((whole[-GUARD:] == FILL).all())


@pytest.mark.parametrize("heads,kv,d", [(4, 4, 128), (6, 2, 64)])
@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("lens,starts,n_tokens", CASES)
def test_attention(fkv, heads, kv, d, workspace, lens, starts, n_tokens):
    x = Paged([(n, 0) for n in lens], 16, kv, d, seed=80)
    b = batch(fkv, x, lens, starts, n_tokens)
    Q = x.rows(heads, d)
    (O, O_all), (lse, lse_all) = guarded((heads, n_tokens, d), BF), guarded((heads, n_tokens), torch.float32)
    ws = ws_all = None
    if workspace:
        ws, ws_all = guarded((-(-fkv.fkv_paged_attention_workspace_size(b, heads, kv, d) // 4),), torch.float32)
        ws = ws.view(torch.uint8)
    fkv.fkv_paged_attention(b, Q.cuda(), x.K.cuda(), x.V.cuda(), 1 / math.sqrt(d), O, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    assert untouched(O_all) and untouched(lse_all) and (ws is None or untouched(ws_all))
    ref, rl, A, top = attend(x, Q, 1 / math.sqrt(d))
    a, e = x.starts[0], x.starts[-1]
    assert close(O.cpu()[:, a:e], ref[:, a:e], A[:, a:e], top[:, a:e], d, max(lens))
    assert close_lse(lse.cpu()[:, a:e], rl[:, a:e], top[:, a:e], d, max(lens))
    for t in (O[:, :a], O[:, e:], lse[:, :a], lse[:, e:]):
        assert bool((t == FILL).all())


@pytest.mark.parametrize("lens,starts,n_tokens", CASES)
def test_append(fkv, lens, starts, n_tokens):
    x = Paged([(n, 0) for n in lens], 16, 2, 64, seed=81)
    b = batch(fkv, x, lens, starts, n_tokens)
    K, V, want = x.rows(2, 64), x.rows(2, 64), [x.K.clone(), x.V.clone()]
    for i, (length, new) in enumerate(x.seqs):
        for t in range(max(new - length, 0), new):
            page, row = x.place(i, length - new + t)
            want[0][page, :, row], want[1][page, :, row] = K[:, x.starts[i] + t], V[:, x.starts[i] + t]
    kp, vp = x.K.cuda(), x.V.cuda()
    fkv.fkv_append_paged(b, K.cuda(), V.cuda(), kp, vp)
    assert torch.equal(kp.cpu(), want[0]) and torch.equal(vp.cpu(), want[1])


@pytest.mark.parametrize("form", ["absorbed", "expanded", "auto"])
@pytest.mark.parametrize("lens,starts,n_tokens", CASES)
def test_latent(fkv, form, lens, starts, n_tokens):
    heads, d, R = 3, 64, 256
    x, _, W_k, W_v = latent_case([(n, 0) for n in lens], 16, heads, d, R, 82)
    b = batch(fkv, x, lens, starts, n_tokens, sum_len=sum(lens))
    Q = x.rows(heads, d + ROT)
    O, O_all = guarded((heads, n_tokens, d), BF)
    ws, ws_all = guarded((-(-fkv.fkv_latent_attention_workspace_size(b, heads, d, R, form) // 4),), torch.float32)
    fkv.fkv_latent_attention(b, Q.cuda(), x.K.cuda(), W_k.cuda(), W_v.cuda(), 1 / math.sqrt(d + ROT), O, form=form,
                             workspace=ws.view(torch.uint8))
    torch.cuda.synchronize()
    assert untouched(O_all) and untouched(ws_all)
    ref, _ = attend_latent(x, Q, W_k, W_v, 1 / math.sqrt(d + ROT))
    a, e = x.starts[0], x.starts[-1]
    assert rel2(O.cpu()[:, a:e], ref[:, a:e]) <= 2.0 ** -7
    assert bool((O[:, :a] == FILL).all()) and bool((O[:, e:] == FILL).all())
