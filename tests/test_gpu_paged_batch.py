"""The paged cache of many sequences on the GPU: its write, attention of new tokens over its
pages, attention over latent rows, against 64 bits."""
import math

import pytest
import torch

from tests.paged_ref import ROT, Paged, attend, attend_latent, close, close_lse, rel2

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


def view(t, layout):
    """A [heads][n][d] GPU copy of t whose memory is [heads][n][d] or [n][heads][d]."""
    return t.cuda() if layout == "head" else t.transpose(0, 1).contiguous().cuda().transpose(0, 1)


def run_attend(fkv, x, Q, causal=True, spans=None, layout="token", workspace=True, fill=7.0, lse=True, scale=None, **kw):
    b = x.batch(fkv, **kw)
    heads, n, d = Q.shape
    q, O = view(Q, layout), view(torch.full((heads, n, d), fill, dtype=BF), layout)
    ls = torch.full((heads, n), fill, device="cuda") if lse else None
    ws = None
    if workspace:
        ws = torch.full((fkv.fkv_paged_attention_workspace_size(b, heads, x.kv, d),), 0xff, dtype=torch.uint8, device="cuda")
    fkv.fkv_paged_attention(b, q, x.K.cuda(), x.V.cuda(), 1 / math.sqrt(d) if scale is None else scale, O, causal=causal,
                            spans=spans, lse=ls, workspace=ws)
    return O.cpu(), None if ls is None else ls.cpu()


def check(x, Q, O, lse, causal, spans, fill=7.0):
    d = Q.shape[2]
    ref, rl, A, top = attend(x, Q, 1 / math.sqrt(d), causal, spans)
    a, b = x.starts[0], x.starts[-1]
    n_keys = max([s[0] for s in x.seqs] + [1])
    assert close(O[:, a:b], ref[:, a:b], A[:, a:b], top[:, a:b], d, n_keys), rel2(O[:, a:b], ref[:, a:b])
    assert close_lse(lse[:, a:b], rl[:, a:b], top[:, a:b], d, n_keys)
    for t in (O[:, :a], O[:, b:]):
        assert bool((t == fill).all())
    if b > a and ref.abs().sum() > 0:         # two independent roundings of at most half a step: 2^-8 / sqrt 3 each
        assert rel2(O[:, a:b], ref[:, a:b]) <= 2.0 ** -8


ONES = [(812, 1), (93, 1), (1, 1), (1300, 1), (64, 1), (65, 1), (33, 1), (257, 1)]
SHORT = [(75, 5), (130, 3), (9, 9), (40, 0), (0, 0), (700, 16)]
LONG = [(300, 300), (61, 61), (1000, 129), (128, 128), (129, 1), (450, 65)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv", [(4, 4), (6, 2), (16, 1)])
@pytest.mark.parametrize("seqs,page,sum_len", [(ONES, 16, None), (SHORT, 48, None), (LONG, 64, None), (LONG, 64, 0)])
def test_causal(fkv, d, heads, kv, seqs, page, sum_len):
    x = Paged(seqs, page, kv, d, seed=d + heads, spare=3, before=2)
    Q = x.rows(heads, d)
    O, lse = run_attend(fkv, x, Q, sum_len=sum_len)
    check(x, Q, O, lse, True, None)


@pytest.mark.parametrize("sum_len", [None, 0])
@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("d,heads,kv,seqs,page,layout", [
    (128, 3, 3, [(1560, 390)], 390, "head"), (64, 2, 1, [(515, 130), (40, 40)], 7, "token"), (128, 2, 2, [(2000, 1)], 1, "head"),
    (64, 5, 1, [(333, 20), (1, 1), (2, 2)], 333, "head")])
def test_chunk(fkv, sum_len, workspace, d, heads, kv, seqs, page, layout):
    x = Paged(seqs, page, kv, d, seed=3)
    Q = x.rows(heads, d)
    O, lse = run_attend(fkv, x, Q, causal=False, layout=layout, workspace=workspace, sum_len=sum_len)
    check(x, Q, O, lse, False, None)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,seqs,sum_len", [(128, ONES, None), (64, SHORT, None), (128, LONG, None), (64, LONG, None), (128, LONG, 0), (64, LONG, 0)])
def test_spans(fkv, causal, d, seqs, sum_len):
    x = Paged(seqs, 32, 4, d, seed=5, spare=1)
    Q = x.rows(8, d)
    spans = [(0, 0), (33, 100), (0, -1), (1, 40)]
    O, lse = run_attend(fkv, x, Q, causal=causal, spans=spans, sum_len=sum_len)
    check(x, Q, O, lse, causal, spans)
    tight = [(4, 64)] * 4                     # no head sees everything
    O, lse = run_attend(fkv, x, Q, causal=causal, spans=tight, sum_len=sum_len)
    check(x, Q, O, lse, causal, tight)


@pytest.mark.parametrize("causal,key", [(True, True), (False, True), (False, False)])
@pytest.mark.parametrize("d,seqs,sum_len", [(64, [(90, 20), (40, 3)], None), (128, [(300, 200), (70, 70)], None), (128, [(300, 200), (70, 70)], 0)])
def test_odd_values_where_not_seen(fkv, causal, key, d, seqs, sum_len):
    """Infinities and NaNs at keys that a row does not see, behind the last token and in other pages."""
    x = Paged(seqs, 16, 2, d, seed=9)
    spans = [(5, 30), (0, -1)]
    for y in range(2):
        for i, (length, new) in enumerate(seqs):
            for t, v in ((length - 2, math.nan), (length - 1, math.inf), (length - new, -math.inf), (7, math.nan)):
                page, row = x.place(i, t)
                x.V[page, y, row, (3 * t + y) % d] = v
                if t == length - 1 and key:
                    x.K[page, y, row, 5] = math.nan
            page, row = x.place(i, length - 1)
            x.K[page, y, row + 1:], x.V[page, y, row + 1:] = math.nan, math.inf
    Q = x.rows(4, d)
    O, lse = run_attend(fkv, x, Q, causal=causal, spans=spans, sum_len=sum_len)
    ref, rl, A, top = attend(x, Q, 1 / math.sqrt(d), causal, spans)
    ref = torch.where(torch.isnan(rl)[..., None], math.nan, ref)
    odd = ~torch.isfinite(ref)
    assert torch.equal(torch.isnan(O.double()), torch.isnan(ref))
    inf = torch.isinf(ref)
    assert torch.equal(O.double()[inf], ref[inf])
    fine = torch.isfinite(rl)
    assert close(torch.where(odd, 0.0, O.double()), torch.where(odd, 0.0, ref), torch.where(odd, 0.0, A), torch.where(fine, top, 0.0), d, 300)
    assert torch.equal(torch.isnan(lse.double()), torch.isnan(rl)) and odd.any()
    assert odd.all() == (key and not causal)   # (the last key's NaN: every row of a chunk sees it)


def run_latent(fkv, x, Q, W_k, W_v, causal=True, span=None, form="auto", layout="token", fill=7.0):
    b = x.batch(fkv)
    heads, n, d = Q.shape[0], Q.shape[1], W_k.shape[1]
    O = view(torch.full((heads, n, d), fill, dtype=BF), layout)
    need = fkv.fkv_latent_attention_workspace_size(b, heads, d, W_k.shape[2], form)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    fkv.fkv_latent_attention(b, view(Q, layout), x.K.cuda(), W_k.cuda(), W_v.cuda(), 1 / math.sqrt(d + ROT), O, causal=causal, span=span,
                             form=form, workspace=ws)
    return O.cpu()


def latent_case(seqs, page, heads, d, R, seed):
    x = Paged(seqs, page, 1, R + ROT, seed=seed, spare=2, before=1, values=False)
    W_k, W_v = ((torch.randn((heads, d, R), generator=x.g) / math.sqrt(R)).to(BF) for _ in range(2))
    return x, x.rows(heads, d + ROT), W_k, W_v


@pytest.mark.parametrize("form", ["absorbed", "expanded", "auto"])
@pytest.mark.parametrize("d,R,heads,seqs,page", [
    (64, 256, 5, SHORT, 16), (128, 512, 12, ONES, 64), (128, 256, 3, [(300, 200), (61, 61), (700, 1)], 48),
    (64, 512, 40, [(70, 1), (400, 2), (140, 130)], 100)])
def test_latent(fkv, form, d, R, heads, seqs, page):
    x, Q, W_k, W_v = latent_case(seqs, page, heads, d, R, 21)
    O = run_latent(fkv, x, Q, W_k, W_v, form=form)
    ref, A = attend_latent(x, Q, W_k, W_v, 1 / math.sqrt(d + ROT))
    a, b = x.starts[0], x.starts[-1]
    # four independent roundings of at most half a step, 2^-8 / sqrt 3 each (the scores' through the absorbed
    # queries or expanded keys moves a probability by as much as the score, of order one)
    assert rel2(O[:, a:b], ref[:, a:b]) <= 2.0 ** -7
    assert bool((O[:, :a] == 7).all()) and bool((O[:, b:] == 7).all())


@pytest.mark.parametrize("form", ["absorbed", "expanded"])
@pytest.mark.parametrize("causal,span", [(True, (33, 100)), (False, (0, 20)), (False, None), (True, (5, 0))])
def test_latent_spans(fkv, form, causal, span):
    x, Q, W_k, W_v = latent_case([(500, 40), (90, 90), (1, 1), (260, 3)], 32, 3, 128, 256, 4)
    O = run_latent(fkv, x, Q, W_k, W_v, causal=causal, span=span, form=form, layout="head")
    ref, A = attend_latent(x, Q, W_k, W_v, 1 / math.sqrt(128 + ROT), causal, span)
    a, b = x.starts[0], x.starts[-1]
    assert rel2(O[:, a:b], ref[:, a:b]) <= 2.0 ** -7


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("heads,d,seqs,page,layout", [
    (4, 64, ONES, 16, "token"), (3, 128, SHORT, 7, "head"), (12, 128, [(1560, 390)], 390, "token"), (1, 320, LONG, 64, "token")])
def test_append(fkv, dtype, heads, d, seqs, page, layout):
    x = Paged(seqs, page, heads, d, seed=2, spare=2, before=1, dtype=dtype, values=d != 320)
    K, V = x.rows(heads, d, dtype), x.rows(heads, d, dtype)
    want = [x.K.clone()] + ([x.V.clone()] if x.V is not None else [])
    for i, (length, new) in enumerate(seqs):
        for t in range(new):
            page_i, row = x.place(i, length - new + t)
            for w, r in zip(want, (K, V)):
                w[page_i, :, row] = r[:, x.starts[i] + t]
    kp, vp = x.K.cuda(), None if x.V is None else x.V.cuda()
    fkv.fkv_append_paged(x.batch(fkv), view(K, layout), None if vp is None else view(V, layout), kp, vp)
    assert torch.equal(kp.cpu(), want[0]) and (vp is None or torch.equal(vp.cpu(), want[1]))
