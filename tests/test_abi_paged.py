"""Refusals of the paged cache's entry points, on the host: every invalid argument is turned
down with the documented status before any device work (no GPU is needed)."""
import ctypes
import math
import os

import pytest

FAKE = 0x1000          # 16-byte aligned, never dereferenced: validation fails first
ARG, SHAPE, CAPACITY = 1, 2, 3


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    if not os.path.exists(m.LIB_PATH):
        from paper_2605_09681_amd import build
        build.build()
    m.lib()
    return m


def _batch(fkv, **kw):
    v = dict(n_seqs=2, max_pages=4, page_tokens=16, n_pages=9, n_tokens=6, max_new=4, sum_len=70, page_table=FAKE,
             seq_len=FAKE, q_start=FAKE)
    v.update(kw)
    return fkv.fkv_batch(**v)


def _rows(fkv, data=FAKE, head=128, token=512):
    return ctypes.byref(fkv.fkv_rows(data, head, token))


def _append(fkv, batch="default", heads=4, d=128, dtype=0, K="default", V="default", Kp=FAKE, Vp=FAKE):
    b = _batch(fkv) if batch == "default" else batch
    K = _rows(fkv) if K == "default" else K
    V = _rows(fkv) if V == "default" else V
    return fkv.lib().fkv_append_paged(None if b is None else ctypes.byref(b), heads, d, dtype, K, V, Kp, Vp, None)


def _attend(fkv, batch="default", heads=4, kv=2, d=128, Q="default", Kp=FAKE, Vp=FAKE, causal=1, spans=None, scale=0.1, O="default",
            lse=None, ws=None, n=0):
    b = _batch(fkv) if batch == "default" else batch
    Q = _rows(fkv) if Q == "default" else Q
    O = _rows(fkv) if O == "default" else O
    return fkv.lib().fkv_paged_attention(None if b is None else ctypes.byref(b), heads, kv, d, Q, Kp, Vp, causal, spans, scale, O,
                                         lse, ws, n, None)


def _latent(fkv, batch="default", heads=4, d=128, R=256, Q="default", pages=FAKE, Wk=FAKE, Wv=FAKE, causal=1, span=None, scale=0.1,
            O="default", form=0, ws=FAKE, n=1 << 40):
    b = _batch(fkv) if batch == "default" else batch
    Q = _rows(fkv, head=192, token=768) if Q == "default" else Q
    O = _rows(fkv) if O == "default" else O
    return fkv.lib().fkv_latent_attention(None if b is None else ctypes.byref(b), heads, d, R, Q, pages, Wk, Wv, causal, span, scale,
                                          O, form, ws, n, None)


@pytest.mark.parametrize("call", [_append, _attend, _latent])
def test_batches(fkv, call):
    assert call(fkv, batch=None) == ARG and "batch" in fkv.fkv_last_error()
    for kw in (dict(n_seqs=0), dict(n_seqs=1025), dict(n_tokens=-1), dict(n_tokens=(1 << 24) + 1), dict(page_tokens=0),
               dict(page_tokens=(1 << 20) + 1), dict(n_pages=0), dict(max_pages=0), dict(n_pages=1 << 30)):
        assert call(fkv, batch=_batch(fkv, **kw)) == SHAPE, kw
    for kw in (dict(max_new=0), dict(sum_len=-1), dict(page_table=None), dict(seq_len=None), dict(q_start=None),
               dict(page_table=FAKE + 2), dict(seq_len=FAKE + 1), dict(q_start=FAKE + 2)):
        assert call(fkv, batch=_batch(fkv, **kw)) == ARG, kw
    # nothing to do
    assert call(fkv, batch=_batch(fkv, n_tokens=0, page_table=None, seq_len=None, q_start=None)) == 0


def test_append(fkv):
    assert _append(fkv, dtype=2) == ARG
    assert _append(fkv, heads=0) == SHAPE and _append(fkv, heads=65) == SHAPE
    for d in (0, -8, 4, 12, 8200):
        assert _append(fkv, d=d) == SHAPE, d
    assert _append(fkv, d=4104, dtype=1) == SHAPE                  # 16416 bytes
    assert _append(fkv, K=None) == ARG and _append(fkv, K=_rows(fkv, data=None)) == ARG
    assert _append(fkv, V=None) == ARG and _append(fkv, Vp=None) == ARG and _append(fkv, Kp=None) == ARG
    assert _append(fkv, Kp=FAKE + 8) == ARG and _append(fkv, Vp=FAKE + 4) == ARG
    for kw in (dict(data=FAKE + 8), dict(head=-128), dict(token=-512), dict(head=4), dict(token=516), dict(token=1 << 37)):
        assert _append(fkv, K=_rows(fkv, **kw)) == ARG and _append(fkv, V=_rows(fkv, **kw)) == ARG, kw


def test_attention(fkv):
    for heads, kv, d in ((0, 1, 128), (65, 1, 128), (4, 0, 128), (4, 3, 128), (2, 4, 128), (4, 2, 96), (4, 2, 256)):
        assert _attend(fkv, heads=heads, kv=kv, d=d) == SHAPE, (heads, kv, d)
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert _attend(fkv, scale=scale) == ARG and _latent(fkv, scale=scale) == ARG
    assert _attend(fkv, causal=2) == ARG and _latent(fkv, causal=-1) == ARG
    for sink, recent in ((-1, 4), (0, -2)):
        spans = (fkv.fkv_span * 2)(fkv.fkv_span(0, -1), fkv.fkv_span(sink, recent))
        assert _attend(fkv, spans=spans) == ARG and "spans[1]" in fkv.fkv_last_error()
        assert _latent(fkv, span=(fkv.fkv_span * 1)(fkv.fkv_span(sink, recent))) == ARG
    assert _attend(fkv, Q=None) == ARG and _attend(fkv, O=None) == ARG and _attend(fkv, Kp=None) == ARG and _attend(fkv, Vp=None) == ARG
    assert _attend(fkv, Kp=FAKE + 8) == ARG and _attend(fkv, Vp=FAKE + 8) == ARG and _attend(fkv, lse=FAKE + 2) == ARG
    assert _attend(fkv, Q=_rows(fkv, token=4)) == ARG
    for kw in (dict(head=64), dict(token=64), dict(head=0)):       # rows of the output that overlap
        assert _attend(fkv, O=_rows(fkv, **kw)) == ARG and "overlap" in fkv.fkv_last_error(), kw


def test_latent(fkv):
    for heads, d, R in ((0, 128, 256), (65, 128, 256), (4, 96, 256), (4, 128, 384), (4, 128, 576)):
        assert _latent(fkv, heads=heads, d=d, R=R) == SHAPE, (heads, d, R)
    assert _latent(fkv, form=3) == ARG and _latent(fkv, form=-1) == ARG
    for name in ("pages", "Wk", "Wv", "ws"):
        assert _latent(fkv, **{name: None}) == ARG and _latent(fkv, **{name: FAKE + 8}) == ARG, name
    assert _latent(fkv, ws=FAKE + 128) == ARG
    assert _latent(fkv, Q=_rows(fkv, token=100)) == ARG and _latent(fkv, O=_rows(fkv, token=64)) == ARG
    assert _latent(fkv, batch=_batch(fkv, sum_len=(1 << 30) + 1)) == SHAPE
    assert _latent(fkv, batch=_batch(fkv, sum_len=1 << 25), form=2) == SHAPE      # 2^17 blocks of 256 tokens


def test_latent_keys_of_4_gib(fkv):
    """2^32 / 384 = 11184810.7 tokens of 192 channels, and the blocks that the sequences may leave unfilled."""
    assert _latent(fkv, d=128, batch=_batch(fkv, sum_len=11_184_800), form=2) == SHAPE


def test_sizes_without_a_device_are_checked_first(fkv):
    out = ctypes.c_size_t(0)
    L = fkv.lib()
    assert L.fkv_paged_attention_workspace_size(None, 4, 2, 128, ctypes.byref(out)) == ARG
    assert L.fkv_paged_attention_workspace_size(ctypes.byref(_batch(fkv)), 4, 3, 128, ctypes.byref(out)) == SHAPE
    assert L.fkv_paged_attention_workspace_size(ctypes.byref(_batch(fkv)), 4, 2, 128, None) == ARG
    assert L.fkv_latent_attention_workspace_size(ctypes.byref(_batch(fkv)), 4, 128, 300, 0, ctypes.byref(out)) == SHAPE
    assert L.fkv_latent_attention_workspace_size(ctypes.byref(_batch(fkv)), 4, 128, 256, 7, ctypes.byref(out)) == ARG
    assert L.fkv_latent_attention_workspace_size(ctypes.byref(_batch(fkv)), 4, 128, 256, 0, None) == ARG


def test_binding(fkv):
    import torch
    cpu = torch.zeros((2, 4), dtype=torch.int32)
    with pytest.raises(ValueError):
        fkv.PagedBatch(cpu, cpu[:, 0], torch.zeros(3, dtype=torch.int32), 16, 4, 4)
    with pytest.raises(TypeError):
        fkv.fkv_append_paged(object(), cpu, cpu, cpu, cpu)
    with pytest.raises(ValueError):
        fkv._spans([(0, 1)], 2)
    with pytest.raises(ValueError):
        fkv._spans([(0, 1 << 40)], 1)
    with pytest.raises(ValueError):
        fkv._form("both")


def test_streams_in_a_step(fkv):
    from paper_2605_09681_amd.layer import PagedStreams
    p = PagedStreams(1, 1, 64, n_pages=4, page_tokens=16, device="cpu")
    streams = [p.open() for _ in range(fkv.FKV_MAX_SEQS + 1)]
    for new in ([], [(streams[0], 0)], [(streams[0], 1)] * 2, [(s, 1) for s in streams]):
        with pytest.raises(ValueError):
            p.step(new)
    with pytest.raises(RuntimeError):
        p.step([(streams[0], 65)])
    assert all(p.length(s) == 0 for s in streams) and len(p._free) == 4
