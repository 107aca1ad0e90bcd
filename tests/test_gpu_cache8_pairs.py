"""Channel pairs that no position axis turns: they stay as they are, bit for bit,
whatever lies in them and beside them, under both pairings and in every output."""
import math

import pytest
import torch

from tests.cache8_ref import Rope, quantise

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BITS = {"bf16": torch.int16, "f32": torch.int32}
D, F, HEADS = 64, 40, 2
TURNED = 10                                          # of 32 pairs


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


def _channels(pair, halves):
    return (pair, pair + D // 2) if halves else (2 * pair, 2 * pair + 1)


def _input(dtype, halves):
    """Random rows; in pairs that stay, one channel is an infinity, a NaN or a zero of either sign beside a
    number of either sign, or both are."""
    x = torch.randn((HEADS, F, D), generator=torch.Generator().manual_seed(1)).to(DT[dtype])
    odd = [math.inf, -math.inf, math.nan, -0.0, 0.0]
    for i, pair in enumerate(range(TURNED, D // 2)):
        a, b = _channels(pair, halves)
        x[0, i, a], x[0, i + 1, b] = odd[i % 5], odd[i % 5]
        x[1, i, a], x[1, i, b] = odd[i % 5], odd[(i + 1) % 5]
        x[1, i + 1, a], x[1, i + 1, b] = -0.0, -1.0
    return x


def _kept(halves):
    stay = torch.zeros(D, dtype=torch.bool)
    for pair in range(TURNED, D // 2):
        stay[list(_channels(pair, halves))] = True
    return stay


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotation_leaves_the_other_pairs(fkv, dtype, halves):
    rope = Rope(5, 3, 2, row_tokens=8, halves=halves).make(fkv)
    shape = fkv.make_shape(HEADS, D, F, 0, 3, 1, F, dtype)
    x, stay = _input(dtype, halves), _kept(halves)
    out = torch.empty_like(x).cuda()
    fkv.fkv_rotate_chunk(shape, rope, [7], None, x.cuda(), None, None, out, None)
    hist = [torch.zeros((HEADS, 3, F, D), dtype=DT[dtype], device="cuda") for _ in range(2)]
    fkv.fkv_append_frames_rotated(shape, rope, [7], x.cuda(), x.cuda(), [1], *hist)
    for got in (out.cpu(), hist[0][:, 1].cpu()):
        assert torch.equal(got[..., stay].view(BITS[dtype]), x[..., stay].view(BITS[dtype]))
        assert bool(got[..., ~stay].isfinite().all())           # nothing reaches the turned pairs


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_8_bit_write_leaves_the_other_pairs(fkv, dtype, halves):
    """An infinity or a NaN in a pair that stays becomes NaN and its partner keeps the code it has alone."""
    rope = Rope(5, 3, 2, row_tokens=8, halves=halves).make(fkv)
    shape = fkv.make_shape(HEADS, D, F, 0, 1, 1, F, dtype)
    x, stay = _input(dtype, halves), _kept(halves)
    # one large element that does not turn sets every block's scale, so the codes of what stays do not
    # depend on the turned channels' roundings
    big = _channels(D // 2 - 1, halves)[1]
    x[:, ::16, big] = 100.0
    cache = fkv.Cache8.zeros(shape, 16)
    fkv.fkv_append_frames_q8(shape, rope, [7], x.cuda(), x.cuda(), [0], cache)
    want, scales = quantise(x.float()[:, None], 16)
    assert torch.equal(cache.k_scale.cpu(), scales)
    got, want = (c.cpu().reshape(x.shape)[..., stay] for c in (cache.K, want))
    spoiled = want.float().isnan()
    assert torch.equal(got.float().isnan(), spoiled)
    assert torch.equal(got.view(torch.uint8)[~spoiled], want.view(torch.uint8)[~spoiled])
    assert not bool(cache.K.cpu().reshape(x.shape)[..., ~stay].float().isnan().any())
