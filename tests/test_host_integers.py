"""Whole numbers that reach the library as 32-bit integers: what does not fit, or is no
whole number, is refused by the binding and not cut down to another slot, position or
size (no GPU is needed)."""
import numpy as np
import pytest
import torch

import paper_2605_09681_amd as fkv

BAD = [1 << 32, (1 << 31), -(1 << 31) - 1, -(1 << 32) + 1, 1.5, float("nan"), float("inf")]


@pytest.mark.parametrize("bad", BAD)
def test_refused(bad):
    refused = pytest.raises((ValueError, OverflowError))
    with refused:
        fkv._ints([0, bad], 2, "dst_slot")
    with refused:
        fkv._slots([bad, 1], 2)
    with refused:
        fkv._positions([3, bad], 2)
    with refused:
        fkv.make_shape(2, 128, 64, 4, 4, 2, bad, "bf16")
    with refused:
        fkv.make_heads([(0, 1, bad, 0, 1)])
    with refused:
        fkv.make_rope(22, 21, bad)
    shape = fkv.make_shape(1, 128, 64, 4, 4, 2, 64, "bf16")
    heads = fkv.make_heads([(0, 1, 1, 0, 1)])
    with refused:
        fkv.fkv_kept_tokens_max(shape, heads, bad)
    with refused:
        fkv.fkv_chunk_attention_q8_workspace_size(shape, heads, bad, 0)
    with refused:
        fkv.fkv_chunk_attention_q8_workspace_size(shape, heads, 1, bad)


def test_taken():
    top, low = (1 << 31) - 1, -(1 << 31)
    for values in ([0, top, low], (0, top, low), np.array([0, top, low]), torch.tensor([0, top, low]),
                   [np.int64(0), np.int32(top), low], iter([0, top, low])):
        assert list(fkv._ints(values, 3, "slots")) == [0, top, low]
    assert list(fkv._slots(None, 3)) == [0, 1, 2]
    assert list(fkv._slots(range(2, 5), 3)) == [2, 3, 4]
    assert len(fkv._ints([], 0, "slots")) == 1
    with pytest.raises(ValueError):
        fkv._ints([1], 2, "slots")
    assert fkv.make_shape(np.int64(2), 128, 64, 4, 4, 2, 64, "bf16").n_heads == 2
