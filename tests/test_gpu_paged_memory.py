"""Memory that PagedStreams holds beside its pages: one workspace, whatever the streams have grown to; smaller ones stay
only where a captured graph uses them."""
import math

import pytest
import torch

from tests.paged_ref import ROT

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
HEADS, D, R, NEW = 12, 128, 256, 300


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


def latent_streams(n_pages=100):
    from paper_2605_09681_amd.layer import PagedStreams
    return PagedStreams(1, HEADS, D, n_pages=n_pages, page_tokens=64, latent_dim=R)


def rows(heads, n, width, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((heads, n, width), generator=g, device="cuda").to(BF)


def weights():
    return [(rows(HEADS, D, R, k) / math.sqrt(R)).contiguous() for k in (1, 2)]


def test_streams_that_grow_by_chunks(fkv):
    """Each chunk's expanded keys need more than the last one's: what is outgrown is freed."""
    p, W = latent_streams(), weights()
    s = p.open()
    K, Q = rows(1, NEW, R + ROT, 3), rows(HEADS, NEW, D + ROT, 4)
    O = torch.empty((HEADS, NEW, D), dtype=BF, device="cuda")
    torch.cuda.synchronize()
    before, sizes = torch.cuda.memory_allocated(), []
    for chunk in range(20):
        b = p.step([(s, NEW)])
        sizes.append(fkv.fkv_latent_attention_workspace_size(b, HEADS, D, R))
        p.append(0, b, K)
        p.attend(0, b, Q, O, W_k=W[0], W_v=W[1])
        torch.cuda.synchronize()
        assert torch.cuda.memory_allocated() - before <= max(sizes) * 3 // 2 + (1 << 20), chunk
    # (beside the parts, which are of one size: 6000 tokens take 22 blocks of 256 more than 300, 2 d + 64 channels a head)
    assert max(sizes) - sizes[0] == 22 * 256 * HEADS * (2 * D + ROT) * 2 and sum(sizes) > 10 * max(sizes)


def test_graph_keeps_its_workspace(fkv):
    """A captured step replays right after larger calls, on its own and on another stream, have outgrown its workspace."""
    p, W = latent_streams(300), weights()
    s, t = p.open(), p.open()
    K, Q = rows(1, NEW, R + ROT, 5), rows(HEADS, NEW, D + ROT, 6)
    b = p.step([(s, NEW)])
    O, big = (torch.empty((HEADS, NEW, D), dtype=BF, device="cuda") for _ in range(2))

    def call():
        p.append(0, b, K)
        p.attend(0, b, Q, O, W_k=W[0], W_v=W[1])
    call()
    torch.cuda.synchronize()
    want, small = O.clone(), p._ws.held.numel()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    before = torch.cuda.memory_allocated()
    for chunk in range(20):
        with torch.cuda.stream(side if chunk % 2 else torch.cuda.current_stream()):
            batch = p.step([(t, NEW)])
            p.append(0, batch, K)
            p.attend(0, batch, Q, big, W_k=W[0], W_v=W[1])
        torch.cuda.synchronize()
    assert p._ws.held.numel() > 2 * small
    assert torch.cuda.memory_allocated() - before <= p._ws.held.numel() + (1 << 20)      # (the graph's own was there)
    junk = torch.full((1 << 24,), 0x7f, dtype=torch.uint8, device="cuda")       # memory that a freed workspace would be
    last = big.clone()
    for _ in range(3):
        O.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want)
        p.attend(0, batch, Q, big, W_k=W[0], W_v=W[1])
        torch.cuda.synchronize()
        assert torch.equal(big, last)
    assert bool((junk == 0x7f).all())
