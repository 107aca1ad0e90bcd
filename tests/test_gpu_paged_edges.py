"""The paged cache's calls at their edges: references that turn out wrong, far scores, many sequences, device data
out of range, workspaces shared and missing, captured graphs, whole runs over many streams."""
import math

import pytest
import torch

from tests.paged_ref import ROT, Paged, attend, attend_latent, close, close_lse, rel2
from tests.test_gpu_paged_batch import BF, check, latent_case, run_attend, run_latent, view

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fkv():
    import paper_2605_09681_amd as m
    m.lib()
    return m


def along(x, Q, levels):
    """Keys of sequence i along a common direction, with scores (in log2 units, before the others') levels[i][j]."""
    d = x.width
    u = torch.zeros(d)
    u[: d // 2] = 1.0
    Q[..., : d // 2] = 1.0
    for i, lv in enumerate(levels):
        for j, level in enumerate(lv):
            page, row = x.place(i, j)
            x.K[page, :, row, : d // 2] = (level * math.log(2.0) * math.sqrt(d) / (d // 2)) * u[: d // 2].to(BF)
    return Q


@pytest.mark.parametrize("sum_len", [None, 0])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,heads,seqs", [(128, 2, [(700, 3)]), (64, 4, [(400, 1), (300, 20)]), (128, 3, [(900, 300)]), (64, 2, [(700, 600)])])
@pytest.mark.parametrize("first,later", [(0.0, 150.0), (150.0, 0.0), (0.0, -400.0), (-300.0, 90.0)])
def test_first_tile_is_a_poor_reference(fkv, sum_len, causal, d, heads, seqs, first, later):
    """Scores that rise or fall by hundreds of log2 units after a part's first tile."""
    x = Paged(seqs, 32, heads, d, seed=1)
    Q = along(x, x.rows(heads, d), [[first if j < 100 else later + 0.05 * (j % 9) for j in range(n)] for n, _ in seqs])
    O, lse = run_attend(fkv, x, Q, causal=causal, sum_len=sum_len)
    check(x, Q, O, lse, causal, None)


@pytest.mark.parametrize("d,seqs", [(128, [(300, 2)]), (64, [(500, 200)])])
@pytest.mark.parametrize("size", [3e3, 1e7, -1e12])
def test_far_scores(fkv, d, seqs, size):
    """Scores far beyond 2^24 log2 units, nearly equal: finite rows, weights by their differences."""
    x = Paged(seqs, 16, 1, d, seed=2)
    Q = torch.zeros((2, x.n_tokens, d), dtype=BF)
    Q[..., 0] = 64.0
    x.K[..., 0] = size / 64.0
    x.K[..., 1:] = 0
    O, lse = run_attend(fkv, x, Q, causal=False, scale=1.0)
    ref, rl, A, top = attend(x, Q, 1.0, False)
    assert torch.isfinite(O).all()
    # all scores of a row are equal: its output is the mean of the values, each product exact
    assert rel2(O, ref) <= 2.0 ** -8
    assert bool(((lse.double() - rl).abs() <= 2.0 ** -22 * rl.abs()).all())


def test_infinite_scores(fkv):
    """Keys whose scores are -infinity weigh nothing; a row of nothing else, or with +infinity, is NaN."""
    x = Paged([(200, 1), (150, 90)], 16, 1, 64, seed=3)
    Q = x.rows(1, 64).abs() + 0.5
    for j in range(0, 150, 3):
        for i in range(2):
            page, row = x.place(i, j)
            x.K[page, 0, row, 0] = -math.inf
    O, lse = run_attend(fkv, x, Q, causal=False)
    check(x, Q, O, lse, False, None)
    page, row = x.place(0, 5)
    x.K[page, 0, row, 0] = math.inf
    O, lse = run_attend(fkv, x, Q, causal=False)
    assert torch.isnan(O[:, :1]).all() and torch.isfinite(O[:, 1:]).all()


@pytest.mark.parametrize("d,kv,heads", [(64, 2, 4), (128, 1, 3)])
def test_many_sequences(fkv, d, kv, heads):
    """More than 64 sequences, of every kind."""
    seqs = [((37 * i) % 400 + n, n) for i, n in enumerate([1, 3, 17, 1, 70, 0, 2, 130] * 17)]
    x = Paged(seqs, 16, kv, d, seed=4, spare=5, before=3)
    Q = x.rows(heads, d)
    for sum_len in (None, 0):
        O, lse = run_attend(fkv, x, Q, sum_len=sum_len)
        check(x, Q, O, lse, True, None)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 12, 16, 21, 32, 33, 48, 64])
def test_groups(fkv, group):
    """Every share of heads to a key head, single tokens and a few."""
    x = Paged([(200, 1), (90, 3), (310, 2), (64, 64)], 24, 1, 64, seed=group)
    Q = x.rows(group, 64)
    O, lse = run_attend(fkv, x, Q)
    check(x, Q, O, lse, True, None)


def test_more_new_tokens_than_tokens(fkv):
    """Rows before position 0 see nothing in a causal call and are not appended."""
    x = Paged([(5, 5), (300, 4)], 16, 2, 64, seed=6)
    b = x.batch(fkv)
    Q = x.rows(4, 64)
    b.seq_len[0] = 3                                     # of 5 new tokens two lie before position 0
    x.seqs = [(3, 5), (300, 4)]
    q, O, lse = view(Q, "token"), torch.full((4, x.n_tokens, 64), 7.0, dtype=BF, device="cuda"), torch.zeros((4, x.n_tokens), device="cuda")
    fkv.fkv_paged_attention(b, q, x.K.cuda(), x.V.cuda(), 0.125, O, lse=lse)
    O, lse = O.cpu(), lse.cpu()
    assert bool((O[:, :2] == 0).all()) and bool((lse[:, :2] == -math.inf).all())
    ref, rl, A, top = attend(x, Q, 0.125)
    assert close(O, ref, A, top, 64, 300) and close_lse(lse, rl, top, 64, 300)
    K = x.rows(2, 64)
    kp, vp = x.K.cuda(), x.V.cuda()
    fkv.fkv_append_paged(b, K.cuda(), K.cuda(), kp, vp)
    want = x.K.clone()
    for i, (length, new) in enumerate(x.seqs):
        for t in range(new):
            if length - new + t >= 0:
                page, row = x.place(i, length - new + t)
                want[page, :, row] = K[:, x.starts[i] + t]
    assert torch.equal(kp.cpu(), want)


def test_device_data_out_of_range(fkv):
    """Lengths, starts and pages out of range are held to it: nothing outside the tensors is read or written."""
    x = Paged([(100, 3), (200, 90), (60, 1)], 16, 2, 64, seed=7, spare=4)
    Q, K = x.rows(4, 64).cuda(), x.rows(2, 64).cuda()
    kp, vp = x.K.cuda(), x.V.cuda()
    ws = None
    for what in ("len", "starts", "pages", "fall"):
        b = x.batch(fkv)
        if what == "len":
            b.seq_len.copy_(torch.tensor([1 << 30, -5, 2 ** 31 - 1], dtype=torch.int32))
        elif what == "starts":
            b.q_start.copy_(torch.tensor([-7, 50, 1 << 30, 3], dtype=torch.int32))
        elif what == "fall":
            b.q_start.copy_(torch.tensor([90, 40, 97, 0], dtype=torch.int32))
        else:
            b.page_table.fill_(1 << 30)
            b.page_table[1] = -9
        before = (kp.clone(), vp.clone())
        if what == "pages":
            fkv.fkv_append_paged(b, K, K, kp, vp)
            assert torch.equal(kp, before[0]) and torch.equal(vp, before[1])
        O = torch.zeros((4, x.n_tokens, 64), dtype=BF, device="cuda")
        ws = torch.empty(fkv.fkv_paged_attention_workspace_size(b, 4, 2, 64), dtype=torch.uint8, device="cuda")
        fkv.fkv_paged_attention(b, Q, kp, vp, 0.125, O, workspace=ws)
        if what == "pages":                              # held to a page of the pool
            assert torch.isfinite(O).all()
    torch.cuda.synchronize()


def test_served_tokens(fkv):
    """Of a sequence with more than max_new new tokens the first max_new are served, the others left as they were."""
    x = Paged([(50, 20), (90, 4)], 16, 1, 64, seed=8)
    Q = x.rows(2, 64)
    O, lse = run_attend(fkv, x, Q, max_new=7)
    ref, rl, A, top = attend(x, Q, 0.125)
    keep = torch.tensor([t < 7 or t >= 20 for t in range(24)])
    assert close(O[:, keep], ref[:, keep], A[:, keep], top[:, keep], 64, 90)
    assert bool((O[:, ~keep] == 7).all())


def test_shared_pages(fkv):
    """Sequences with a common beginning read the same pages."""
    x = Paged([(130, 2), (140, 1)], 32, 2, 128, seed=9)
    x.table[1, :4] = x.table[0, :4]
    Q = x.rows(2, 128)
    O, lse = run_attend(fkv, x, Q)
    check(x, Q, O, lse, True, None)


@pytest.mark.parametrize("d,heads,seqs,form", [(64, 3, [(200, 6), (180, 150)], "absorbed"), (128, 2, [(200, 6), (180, 150)], "expanded")])
def test_latent_odd_values_where_not_seen(fkv, d, heads, seqs, form):
    x, Q, W_k, W_v = latent_case(seqs, 16, heads, d, 256, 31)
    W_v.abs_()                                           # (an infinity in a latent row is one in every value)
    for i, (length, new) in enumerate(seqs):
        page, row = x.place(i, length - 2)
        x.K[page, 0, row, 9] = math.inf
        page, row = x.place(i, length - 1)
        x.K[page, 0, row, 300] = math.nan
        x.K[page, 0, row + 1:] = math.nan
    O = run_latent(fkv, x, Q, W_k, W_v, form=form)
    for i, (length, new) in enumerate(seqs):
        a = x.starts[i]
        cut = Paged.__new__(Paged)
        cut.__dict__.update(x.__dict__, seqs=[(0, 0)] * i + [(length - 2, new - 2)] + [(0, 0)] * (len(seqs) - i - 1),
                            starts=[a] * (i + 1) + [a + new - 2] * (len(seqs) - i))
        ref, _ = attend_latent(cut, Q, W_k, W_v, 1 / math.sqrt(d + ROT))
        assert rel2(O[:, a:a + new - 2], ref[:, a:a + new - 2]) <= 2.0 ** -7
        assert not torch.isfinite(O[:, a + new - 2:a + new]).all(2).any()


def test_latent_first_tile_is_a_poor_reference(fkv):
    x, Q, W_k, W_v = latent_case([(500, 4), (300, 1)], 32, 6, 64, 256, 12)
    Q[..., 64:] = 0
    Q[..., 64] = 8.0
    for i in range(2):
        for j in range(x.seqs[i][0]):
            page, row = x.place(i, j)
            x.K[page, 0, row, 256] = 0.0 if j < 150 else 200.0
    O = run_latent(fkv, x, Q, W_k, W_v, form="absorbed")
    ref, A = attend_latent(x, Q, W_k, W_v, 1 / math.sqrt(64 + ROT))
    a, b = x.starts[0], x.starts[-1]
    assert rel2(O[:, a:b], ref[:, a:b]) <= 2.0 ** -7


def test_latent_room_for_fewer_tokens(fkv):
    """Tokens beyond sum_len are left out of the expanded form, nothing is written behind its room."""
    x, Q, W_k, W_v = latent_case([(900, 200)], 64, 2, 64, 256, 13)
    b = x.batch(fkv, sum_len=100)
    n = fkv.fkv_latent_attention_workspace_size(b, 2, 64, 256, "expanded")
    ws = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    O = torch.zeros((2, x.n_tokens, 64), dtype=BF, device="cuda")
    fkv.fkv_latent_attention(b, Q.cuda(), x.K.cuda(), W_k.cuda(), W_v.cuda(), 0.1, O, form="expanded", workspace=ws[:n])
    assert bool((ws[n:] == 0x5a).all()) and torch.isfinite(O).all()


def test_workspace_shared_by_calls_of_other_sizes(fkv):
    """One workspace, calls of many sizes in turn, then the first again: the same bits."""
    cases = [Paged([(900, 1), (40, 1)], 32, 2, 128, seed=40), Paged([(800, 300)], 32, 2, 128, seed=41),
             Paged([(400, 5), (700, 100)], 32, 2, 128, seed=42)]
    runs = []
    for x in cases:
        b = x.batch(fkv)
        runs.append((b, x.rows(4, 128).cuda(), x.K.cuda(), x.V.cuda(), fkv.fkv_paged_attention_workspace_size(b, 4, 2, 128)))
    ws = torch.full((max(r[4] for r in runs),), 0xff, dtype=torch.uint8, device="cuda")
    outs = []
    for k in (0, 1, 2, 0, 1, 2):
        b, Q, K, V, _ = runs[k]
        O = torch.zeros_like(Q)
        fkv.fkv_paged_attention(b, Q, K, V, 0.1, O, workspace=ws)
        outs.append(O)
    for k in range(3):
        assert torch.equal(outs[k], outs[k + 3])


def test_workspace_too_small(fkv):
    x = Paged([(900, 1)], 32, 2, 128, seed=40)
    b, Q = x.batch(fkv), x.rows(2, 128).cuda()
    n = fkv.fkv_paged_attention_workspace_size(b, 2, 2, 128)
    with pytest.raises(fkv.FkvError) as e:
        fkv.fkv_paged_attention(b, Q, x.K.cuda(), x.V.cuda(), 0.1, torch.zeros_like(Q),
                                workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == fkv.FKV_ERR_CAPACITY


@pytest.mark.parametrize("latent", [False, True])
def test_captured_graph(fkv, latent):
    """A captured step replayed with other lengths, pages and tokens, eager work between the replays."""
    d, R = 64, 256
    seqs = [(300, 3), (200, 3), (130, 3)]
    x = Paged(seqs, 16, 1 if latent else 2, R + ROT if latent else d, seed=50, values=not latent, extra_pages=40)
    x.table = torch.cat([x.table, torch.full((3, 20), -1, dtype=torch.int32)], 1)
    free = [p for p in range(x.n_pages) if p not in set(x.table.flatten().tolist())]
    for i in range(3):
        k = -(-seqs[i][0] // 16)
        x.table[i, k:k + 10] = torch.tensor(free[10 * i:10 * i + 10], dtype=torch.int32)
    b = x.batch(fkv, sum_len=2000)
    heads = 4
    W_k, W_v = ((torch.randn((heads, d, R), generator=x.g) / 16).to(BF) for _ in range(2))
    Q = x.rows(heads, d + ROT if latent else d)
    K, V = x.rows(x.kv, x.width), x.rows(x.kv, x.width)
    q, k_new, v_new, kp, vp = Q.cuda(), K.cuda(), V.cuda(), x.K.cuda(), None if latent else x.V.cuda()
    wk, wv = W_k.cuda(), W_v.cuda()
    O = torch.zeros((heads, x.n_tokens, d), dtype=BF, device="cuda")
    n = fkv.fkv_latent_attention_workspace_size(b, heads, d, R) if latent else fkv.fkv_paged_attention_workspace_size(b, heads, 2, d)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def step():
        fkv.fkv_append_paged(b, k_new, None if latent else v_new, kp, vp)
        if latent:
            fkv.fkv_latent_attention(b, q, kp, wk, wv, 0.1, O, workspace=ws)
        else:
            fkv.fkv_paged_attention(b, q, kp, vp, 0.1, O, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for lens in ([300, 200, 130], [303, 203, 133], [420, 3, 250], [4, 330, 131]):
        b.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        q.normal_(generator=torch.Generator(device="cuda").manual_seed(lens[0]))
        g.replay()
        got = O.clone()
        torch.cuda.synchronize()
        O.fill_(3.0)
        step()
        assert torch.equal(got, O)
        ws.fill_(0xee)
        x.seqs = [(length, 3) for length in lens]
        x.K, x.V = kp.cpu(), None if latent else vp.cpu()
        ref = (attend_latent(x, q.cpu(), W_k, W_v, 0.1) if latent else attend(x, q.cpu(), 0.1))[0]
        assert rel2(got.cpu(), ref) <= 2.0 ** -7


def test_other_stream(fkv):
    x = Paged([(900, 2), (400, 100)], 32, 2, 64, seed=60)
    b, Q, K, V = x.batch(fkv), x.rows(4, 64).cuda(), x.K.cuda(), x.V.cuda()
    ws = torch.empty(fkv.fkv_paged_attention_workspace_size(b, 4, 2, 64), dtype=torch.uint8, device="cuda")
    A, B = torch.zeros_like(Q), torch.zeros_like(Q)
    fkv.fkv_paged_attention(b, Q, K, V, 0.1, A, workspace=ws)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    fkv.fkv_paged_attention(b, Q, K, V, 0.1, B, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(A, B)


@pytest.mark.parametrize("latent", [0, 256])
def test_streams(fkv, latent):
    """Streams that open, read a prompt, answer token by token and close, whose pages then serve others: every
    step of every layer against 64 bits over the tokens that the stream was given."""
    from paper_2605_09681_amd.layer import PagedStreams
    heads, kv, d, layers = 4, 2, 64, 2
    p = PagedStreams(layers, heads, d, n_pages=40, page_tokens=16, n_kv_heads=None if latent else kv, latent_dim=latent)
    width = latent + ROT if latent else d
    g = torch.Generator().manual_seed(77)
    W = [[(torch.randn((heads, d, latent), generator=g) / 16).to(BF) for _ in range(2)] for _ in range(layers)] if latent else None
    given = {}                                            # stream -> per layer the rows given so far
    plan = [[("a", 70), ("b", 9)], [("a", 1), ("b", 1), ("c", 140)], [("b", 1), ("c", 1)], [("c", 1), ("a", 1), ("d", 33), ("b", 5)],
            "close a", [("e", 200), ("d", 1)], [("e", 1), ("c", 2)]]
    ids = {}
    for step in plan:
        if isinstance(step, str):
            p.close(ids.pop(step[-1]))
            continue
        for name, _ in step:
            if name not in ids:
                ids[name] = p.open()
                given[name] = [[[], []] for _ in range(layers)]
        batch = p.step([(ids[name], n) for name, n in step])
        n = batch.n_tokens
        for layer in range(layers):
            rows = lambda h, w: torch.randn((n, h, w), generator=g).to(BF)  # noqa: E731
            K, V, Q = rows(p.kv, width), rows(p.kv, width), rows(heads, d + ROT if latent else d)
            O = torch.zeros((n, heads, d), dtype=BF, device="cuda")
            p.append(layer, batch, K.cuda().transpose(0, 1), None if latent else V.cuda().transpose(0, 1))
            kw = dict(W_k=W[layer][0].cuda(), W_v=W[layer][1].cuda()) if latent else {}
            p.attend(layer, batch, Q.cuda().transpose(0, 1), O.transpose(0, 1), **kw)
            a = 0
            for name, new in step:
                mem = given[name][layer]
                mem[0].append(K[a:a + new])
                mem[1].append(V[a:a + new])
                x = Paged.__new__(Paged)
                k, v = torch.cat(mem[0]).transpose(0, 1), torch.cat(mem[1]).transpose(0, 1)
                x.K, x.V, x.kv, x.page, x.seqs, x.starts = k[None], v[None], p.kv, k.shape[1], [(k.shape[1], new)], [0, new]
                x.table = torch.zeros((1, 1), dtype=torch.int32)
                assert p.length(ids[name]) == k.shape[1]
                q = Q[a:a + new].transpose(0, 1)
                ref = attend_latent(x, q, *W[layer], p.scale)[0] if latent else attend(x, q, p.scale)[0]
                assert rel2(O[a:a + new].cpu().transpose(0, 1), ref) <= 2.0 ** (-7 if latent else -8)
                a += new
    with pytest.raises(RuntimeError):
        p.step([(ids["e"], 10000)])
    with pytest.raises(ValueError):
        p.step([(ids["e"], 1), (ids["e"], 1)])


@pytest.mark.parametrize("new,sum_len", [(1, None), (90, 0)])
def test_pages_past_2_31_elements(fkv, new, sum_len):
    """Pages whose offsets pass 32 bits in elements and in bytes: written, then attended."""
    n_pages, kv, page, d = 22100, 12, 64, 128            # 2.17e9 elements a pool
    seqs = [(150, new)]
    x = Paged(seqs, page, kv, d, seed=70)
    kp, vp = (torch.zeros((n_pages, kv, page, d), dtype=BF, device="cuda") for _ in range(2))
    far = torch.tensor([n_pages - 1, 5, n_pages - 2], dtype=torch.int32)
    for at, to in zip(x.table[0, :3].tolist(), far.tolist()):
        kp[to], vp[to] = x.K[at].cuda(), x.V[at].cuda()
    K, V, Q = x.rows(kv, d), x.rows(kv, d), x.rows(kv, d)
    for t in range(new):
        at, row = x.place(0, 150 - new + t)
        x.K[at, :, row], x.V[at, :, row] = K[:, t], V[:, t]
    b = x.batch(fkv, sum_len=sum_len)
    b.page_table[0, :3] = far.cuda()
    O, lse = torch.zeros((kv, new, d), dtype=BF, device="cuda"), torch.zeros((kv, new), device="cuda")
    ws = torch.empty(fkv.fkv_paged_attention_workspace_size(b, kv, kv, d), dtype=torch.uint8, device="cuda")
    fkv.fkv_append_paged(b, K.cuda(), V.cuda(), kp, vp)
    fkv.fkv_paged_attention(b, Q.cuda(), kp, vp, 1 / math.sqrt(d), O, lse=lse, workspace=ws)
    check(x, Q, O.cpu(), lse.cpu(), True, None)


@pytest.mark.parametrize("seqs", [[(300001, 1)], [(100003, 70)]])
def test_long_sequences(fkv, seqs):
    x = Paged(seqs, 100, 1, 64, seed=71)
    Q = x.rows(2, 64)
    for sum_len in (None, 0):
        O, lse = run_attend(fkv, x, Q, sum_len=sum_len)
        check(x, Q, O, lse, True, None)


@pytest.mark.parametrize("d,sum_len", [(128, 5_800_001), (64, 9_000_001)])
def test_expanded_copies_past_2_31_bytes(fkv, d, sum_len):
    """A sequence whose expanded keys pass 32 bits of offset; rows see its first and its last tokens."""
    R, page, span = 256, 1000, (100, 500)
    pages = -(-sum_len // page)
    near = sum_len - (pages - 3) * page                  # the same last tokens, and the first, of a short sequence
    x, Q, W_k, W_v = latent_case([(page + near, 70)], page, 1, d, R, 72)
    ref, _ = attend_latent(x, Q, W_k, W_v, 1 / math.sqrt(d + ROT), True, span)
    short = x.table[0]
    x.seqs = [(sum_len, 70)]
    x.table = torch.full((1, pages), int(short[0]), dtype=torch.int32)
    x.table[0, -3:] = short[1:4]
    O = run_latent(fkv, x, Q, W_k, W_v, span=span, form="expanded")
    a, b = x.starts
    assert rel2(O[:, a:b], ref[:, a:b]) <= 2.0 ** -7


@pytest.mark.parametrize("causal", [True, False])
def test_latent_room_ends_before_what_a_row_sees(fkv, causal):
    """Rows that only see tokens beyond the room of the expanded form see no key."""
    x, Q, W_k, W_v = latent_case([(900, 200)], 64, 2, 64, 256, 14)
    b = x.batch(fkv, sum_len=0)                          # (256 tokens)
    O = torch.full((2, x.n_tokens, 64), 7, dtype=BF, device="cuda")
    fkv.fkv_latent_attention(b, Q.cuda(), x.K.cuda(), W_k.cuda(), W_v.cuda(), 0.1, O, causal=causal, span=(0, 50), form="expanded")
    assert bool((O[:, x.starts[0]:x.starts[1]] == 0).all())


def test_small_scale(fkv):
    """A scale that makes every probability one: plain means."""
    x = Paged([(2000, 1), (700, 90)], 64, 1, 64, seed=73)
    Q = x.rows(2, 64)
    for sum_len in (None, 0):
        O, lse = run_attend(fkv, x, Q, sum_len=sum_len, scale=1e-42)
        ref, rl, A, top = attend(x, Q, 1e-42)
        assert close(O, ref, A, top, 64, 2000) and close_lse(lse, rl, top, 64, 2000)
