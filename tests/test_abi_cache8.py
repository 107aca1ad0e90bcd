"""Refusals of the rotation and 8-bit cache entry points, on the host: every
invalid argument is turned down with the documented status before any device
work (no GPU is needed)."""
import ctypes
import math
import os

import pytest

import workloads as W

FAKE = 0x1000          # 16-byte aligned, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    if not os.path.exists(m.LIB_PATH):
        from paper_2605_09681_amd import build
        build.build()
    m.lib()
    return m


def _shape(fkv, **kw):
    base = dict(n_heads=2, head_dim=128, frame_tokens=64, hist_frames=4, cap_frames=4, chunk_frames=2, seg_tokens=64,
                dtype="bf16")
    base.update(kw)
    return fkv.make_shape(**base)


def _heads(fkv):
    return fkv.make_heads((W.HeadBudget(W.STATIC, 1, 1), W.HeadBudget(W.DYNAMIC, 0, 0, 2)))


def _ints(*v):
    return (ctypes.c_int32 * max(len(v), 1))(*v)


def _rope(fkv, **kw):
    base = dict(frame_pairs=22, row_pairs=21, col_pairs=21, row_tokens=8)
    base.update(kw)
    return fkv.make_rope(**base)


def _rotate(fkv, shape=None, rope="default", pos=(0, 1), Q=FAKE, Qr=FAKE, strides=(128, 256), K=None, Kr=None):
    shape = _shape(fkv) if shape is None else shape
    rope = _rope(fkv) if rope == "default" else rope
    q = None if Q is None else ctypes.byref(fkv.fkv_rows(Q, *strides))
    k = None if K is None else ctypes.byref(fkv.fkv_rows(K, *strides))
    return fkv.lib().fkv_rotate_chunk(ctypes.byref(shape), None if rope is None else ctypes.byref(rope),
                                      None if pos is None else _ints(*pos), q, k, None, Qr, Kr, None, None)


@pytest.mark.parametrize("kw", [
    dict(frame_pairs=-1), dict(row_pairs=-1), dict(col_pairs=-1), dict(frame_pairs=23), dict(frame_pairs=2 ** 31 - 1),
    dict(row_tokens=0), dict(row_tokens=65), dict(token_step=2), dict(token_step=-1), dict(pairing=2),
    dict(theta=0.5), dict(theta=math.inf), dict(theta=math.nan), dict(theta=-3.0)])
def test_bad_rotations(fkv, kw):
    assert _rotate(fkv, rope=_rope(fkv, **kw)) == 1
    assert fkv.fkv_last_error()


def test_rotate_arguments(fkv):
    far = 1 << 24
    assert _rotate(fkv, rope=None) == 1
    assert _rotate(fkv, pos=None) == 1
    assert _rotate(fkv, pos=(0, far + 1)) == 1 and "frame_pos[1]" in fkv.fkv_last_error()
    assert _rotate(fkv, pos=(-far - 1, 0)) == 1
    assert _rotate(fkv, Q=None, Qr=None) == 1                 # nothing to rotate
    assert _rotate(fkv, Qr=None) == 1 and _rotate(fkv, Q=None) == 1
    assert _rotate(fkv, K=FAKE) == 1 and _rotate(fkv, Kr=FAKE) == 1
    assert _rotate(fkv, Q=FAKE + 8) == 1 and _rotate(fkv, Qr=FAKE + 4) == 1
    for strides in ((-128, 256), (128, -256), (4, 256), (128, 129)):
        assert _rotate(fkv, strides=strides) == 1, strides
    assert _rotate(fkv, shape=_shape(fkv, head_dim=96)) == 2
    assert _rotate(fkv, shape=_shape(fkv, chunk_frames=300, frame_tokens=8, seg_tokens=8), pos=(0,) * 300) == 2


def _append(fkv, n=2, slots=(0, 1), pos=(0, 1), K=FAKE, hist=FAKE, strides=(128, 256)):
    rows = fkv.fkv_rows(K, *strides)
    return fkv.lib().fkv_append_frames_rotated(
        ctypes.byref(_shape(fkv)), ctypes.byref(_rope(fkv)), None if pos is None else _ints(*pos), ctypes.byref(rows),
        ctypes.byref(rows), n, None if slots is None else _ints(*slots), hist, hist, None)


def _append8(fkv, n=2, slots=(0, 1), pos=(0, 1), K=FAKE, cache="default", rope="default", shape=None):
    rows = fkv.fkv_rows(K, 128, 256)
    c = fkv.fkv_cache8(FAKE, FAKE, FAKE, FAKE, 64) if cache == "default" else cache
    rope = _rope(fkv) if rope == "default" else rope
    return fkv.lib().fkv_append_frames_q8(
        ctypes.byref(_shape(fkv) if shape is None else shape), None if rope is None else ctypes.byref(rope),
        None if pos is None else _ints(*pos), ctypes.byref(rows), ctypes.byref(rows), n,
        None if slots is None else _ints(*slots), None if c is None else ctypes.byref(c), None)


@pytest.mark.parametrize("call", [_append, _append8])
def test_append_arguments(fkv, call):
    assert call(fkv, n=0, slots=(), pos=()) == 0              # nothing to write
    assert call(fkv, n=5, slots=(0, 1, 2, 3, 0), pos=(0,) * 5) == 1
    assert call(fkv, n=-1) == 1
    assert call(fkv, slots=(1, 1)) == 1 and "twice" in fkv.fkv_last_error()
    assert call(fkv, slots=(1, 4)) == 1 and call(fkv, slots=(-1, 0)) == 1
    assert call(fkv, slots=None) == 1 and call(fkv, pos=None) == 1
    assert call(fkv, pos=(0, 1 << 25)) == 1
    assert call(fkv, K=None) == 1 and call(fkv, K=FAKE + 2) == 1


def test_append_rotated_destination(fkv):
    assert _append(fkv, hist=None) == 1 and _append(fkv, hist=FAKE + 8) == 1
    assert _append(fkv, strides=(128, 132)) == 1


@pytest.mark.parametrize("fields", [
    (FAKE, FAKE, FAKE, FAKE, 0), (FAKE, FAKE, FAKE, FAKE, 48), (FAKE, FAKE, FAKE, FAKE, 256), (FAKE, FAKE, FAKE, FAKE, 8),
    (None, FAKE, FAKE, FAKE, 64), (FAKE, None, FAKE, FAKE, 64), (FAKE, FAKE, None, FAKE, 64),
    (FAKE, FAKE, FAKE, None, 64), (FAKE + 8, FAKE, FAKE, FAKE, 64), (FAKE, FAKE + 8, FAKE, FAKE, 64)])
def test_bad_caches(fkv, fields):
    bad = fkv.fkv_cache8(*fields)
    assert _append8(fkv, cache=bad) == 1
    assert _attend(fkv, cache=bad) == 1


def test_append8_arguments(fkv):
    assert _append8(fkv, cache=None) == 1
    assert _append8(fkv, rope=None, pos=None, K=None) == 1    # frame_pos is not needed then, K is
    assert _append8(fkv, shape=_shape(fkv, head_dim=32)) == 2


def _score(fkv, shape=None, cache="default", slots=(0, 1, 2, 3), K=FAKE, scores=FAKE, kept=FAKE, kv=FAKE, ws=FAKE, short=0):
    shape = _shape(fkv) if shape is None else shape
    heads = _heads(fkv)
    need = fkv.fkv_score_workspace_size(shape, heads)
    c = fkv.fkv_cache8(FAKE, FAKE, FAKE, FAKE, 64) if cache == "default" else cache
    return fkv.lib().fkv_score_select_q8(ctypes.byref(shape), heads, None if c is None else ctypes.byref(c), _ints(*slots),
                                         K, scores, kept, kv, ws, need - short, None)


def test_score_arguments(fkv):
    assert _score(fkv, shape=_shape(fkv, dtype="f32")) == 2
    assert _score(fkv, cache=None) == 1
    assert _score(fkv, cache=fkv.fkv_cache8(FAKE, FAKE, FAKE, FAKE, 20)) == 1
    assert _score(fkv, cache=fkv.fkv_cache8(None, FAKE, FAKE, FAKE, 64)) == 1
    assert _score(fkv, slots=(0, 1, 2, 4)) == 1
    for name in ("K", "scores", "kept", "kv", "ws"):
        assert _score(fkv, **{name: None}) == 1, name
    assert _score(fkv, K=FAKE + 8) == 1
    assert _score(fkv, short=1) == 3


def _attend(fkv, shape=None, cache="default", slots=(0, 1, 2, 3), kept=FAKE, kv=FAKE, Q=FAKE, n_q=4, K=FAKE, n_cur=3,
            scale=0.1, O=FAKE, heads=None):
    shape = _shape(fkv) if shape is None else shape
    c = fkv.fkv_cache8(FAKE, FAKE, FAKE, FAKE, 64) if cache == "default" else cache
    return fkv.lib().fkv_chunk_attention_q8(
        ctypes.byref(shape), _heads(fkv) if heads is None else heads, None if c is None else ctypes.byref(c),
        None if slots is None else _ints(*slots), kept, kv, Q, n_q, K, K, n_cur, ctypes.c_float(scale), O, None, None, 0,
        None)


def test_attention_arguments(fkv):
    assert _attend(fkv, shape=_shape(fkv, dtype="f32")) == 2
    assert _attend(fkv, cache=None) == 1
    assert _attend(fkv, n_q=0) == 1 and _attend(fkv, n_q=-4) == 1 and _attend(fkv, n_cur=-1) == 1
    assert _attend(fkv, n_q=1 << 23) == 2 and _attend(fkv, n_cur=1 << 23) == 2     # 2^31 bytes of rows
    assert _attend(fkv, slots=None) == 1 and _attend(fkv, slots=(0, 1, 2, 7)) == 1
    for name in ("kept", "kv", "Q", "K", "O"):
        assert _attend(fkv, **{name: None}) == 1, name
    for name in ("Q", "K", "O"):
        assert _attend(fkv, **{name: FAKE + 8}) == 1, name
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert _attend(fkv, scale=scale) == 1, scale
    many = fkv.make_shape(64, 64, 64, 4, 4, 1, 64, "bf16")     # more query tiles than one launch holds
    heads = fkv.make_heads([W.HeadBudget(W.STATIC, 1, 1)] * 64)
    assert _attend(fkv, shape=many, heads=heads, n_q=1 << 22, K=None, n_cur=0) == 2
    bad = fkv.make_heads((W.HeadBudget(W.STATIC, -1, 1), W.HeadBudget(W.DYNAMIC, 0, 0, 2)))
    assert _attend(fkv, heads=bad) == 1
    size = ctypes.c_size_t(0)
    query = fkv.lib().fkv_chunk_attention_q8_workspace_size
    shape = _shape(fkv)
    assert query(ctypes.byref(shape), _heads(fkv), 0, 0, ctypes.byref(size)) == 1
    assert query(ctypes.byref(shape), _heads(fkv), 1, 0, None) == 1


def test_binding_refusals(fkv):
    """The Python layer's own checks (tensors on the host are refused before anything else)."""
    import torch
    shape, rope = _shape(fkv), _rope(fkv)
    x = torch.zeros((2, 128, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        fkv.fkv_rotate_chunk(shape, rope, [0, 1], x, None, None, x, None, None)          # CPU tensors
    with pytest.raises(ValueError):
        fkv._positions([0], 2)                                                            # one position for two frames
    with pytest.raises(ValueError):
        fkv._positions([0, 1 << 25], 2)
    with pytest.raises(ValueError):
        fkv.fkv_rotate_chunk(shape, rope, [0, 1], None, None, None, None, None, None)
    with pytest.raises(ValueError):
        fkv.fkv_rotate_chunk(shape, rope, [0, 1], x, None, None, None, None, None)
    with pytest.raises(TypeError):
        fkv._cache8(shape, object(), 0)
    with pytest.raises(ValueError):
        fkv._cache8(shape, fkv.Cache8.zeros(shape, 64, device="cpu"), 0)                  # CPU tensors
    bad = fkv.Cache8.zeros(shape, 64, device="cpu")
    bad.block_tokens = 20
    with pytest.raises(ValueError):
        fkv._cache8(shape, bad, 0)
