"""How the paged calls deal a batch to workgroups, on the host: the library's own plan and the
kernels' own code for sequences, splits and owners (tests/paged_host.cpp), over lengths and starts
in any order.  Whatever the batch holds, a row belongs to one sequence at most, every part of a
cut item has a workgroup, and slots and joins stay inside what the workspace has room for."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2605_09681_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
I32 = ctypes.c_int32


class Batch(ctypes.Structure):
    _fields_ = [("n_seqs", I32), ("max_pages", I32), ("page_tokens", I32), ("n_pages", I32), ("n_tokens", I32), ("max_new", I32),
                ("sum_len", ctypes.c_int64), ("page_table", ctypes.c_void_p), ("seq_len", ctypes.c_void_p), ("q_start", ctypes.c_void_p)]


class Span(ctypes.Structure):
    _fields_ = [("sink", I32), ("recent", I32)]


class Item(ctypes.Structure):
    _fields_ = [(n, I32) for n in "seq start n len first y rt part parts slot step join".split()]


class Plan(ctypes.Structure):
    _fields_ = [(n, I32) for n in "rows n_work n_slots n_joins lo hi count tiles".split()]


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    """The host build of tests/paged_host.cpp."""
    try:
        cc = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.hipcc()))), "llvm", "bin", "clang++")
    except RuntimeError:
        pytest.skip("needs hipcc")
    if not os.path.exists(cc):
        cc = os.path.join("/opt/rocm", "llvm", "bin", "clang++")
    so = str(tmp_path_factory.mktemp("paged") / "paged_host.so")
    r = subprocess.run([cc, "-x", "c++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__",
                        "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.dirname(cc))), "include"),
                        "-I", os.path.join(build.ROOT, "include"), "-I", os.path.join(build.PKG, "csrc"),
                        os.path.join(HERE, "paged_host.cpp"), "-o", so], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    L = ctypes.CDLL(so)
    B = ctypes.POINTER(Batch)
    L.host_attend.argtypes = [B, I32, I32, I32, ctypes.POINTER(Span), I32]
    L.host_latent.argtypes = [B, I32, I32, I32, I32]
    L.host_append.argtypes = [B, I32, I32, I32, I32]
    L.host_plan.restype = ctypes.POINTER(Plan)
    return L


class Case:
    def __init__(self, lens, starts, n_tokens, max_new=None, sum_len=0, pages=1 << 15, page=16):
        self.lens, self.starts, self.n_tokens = lens, starts, n_tokens
        self.max_new = n_tokens if max_new is None else max_new
        self._arrays = (I32 * len(lens))(*lens), (I32 * len(starts))(*starts), (I32 * 1)()
        at = [ctypes.addressof(a) for a in self._arrays]
        self.c = Batch(len(lens), pages, page, 1, n_tokens, self.max_new, sum_len, at[2], at[0], at[1])

    def rows(self):
        """Each sequence's first row, new tokens and position of the first of them: starts are held to the batch's rows, and
        to the largest start before them."""
        out, at = [], 0
        for i in range(len(self.lens)):
            at = max(at, min(max(self.starts[i], 0), self.n_tokens))
            end = max(at, min(max(self.starts[i + 1], 0), self.n_tokens))
            length = min(max(self.lens[i], 0), self.c.max_pages * self.c.page_tokens)
            out.append((at, min(end - at, self.max_new), length - (end - at)))
        return out


def read(fn, kind, width=1):
    p = ctypes.POINTER(kind)()
    n = fn(ctypes.byref(p))
    return [p[k] for k in range(n * width)]


def check(L, case, group, kv):
    """The launch for few rows, as the workgroups see it."""
    p, want = L.host_plan().contents, case.rows()
    if p.rows == 0:
        return
    work = read(L.host_items, Item)
    parts, joins, slots = {}, {}, set()
    for w in work:
        start, n, first = want[w.seq]
        assert (w.start, w.n, w.first) == (start, n, first) and p.lo <= n <= p.hi
        assert 0 <= w.y < kv and 0 <= w.rt < -(-n * group // p.rows) and 0 <= w.part < w.parts
        key = (w.seq, w.y, w.rt)
        assert w.part not in parts.setdefault(key, set())
        parts[key].add(w.part)
        if w.parts > 1:
            slot = w.slot + w.part * w.step
            assert 0 <= slot < p.n_slots and slot not in slots
            slots.add(slot)
            assert joins.setdefault(w.join, (key, w.slot, w.step, w.parts)) == (key, w.slot, w.step, w.parts)
    items = {(i, y, rt) for i, (_, n, _) in enumerate(want) if n > 0 and p.lo <= n <= p.hi for y in range(kv)
             for rt in range(-(-n * group // p.rows))}
    assert set(parts) == items                             # every item has its workgroups,
    for w in work:
        assert len(parts[w.seq, w.y, w.rt]) == w.parts     # one for every part
    assert p.count <= p.n_joins and sorted(joins) == list(range(p.count))


FALLING = [
    # every second sequence claims all rows of the batch
    (64, [1] * 1023 + [100000], [0, 64] * 512 + [0]),
    (64, [1] * 1022 + [100000, 1], [64, 0] * 512 + [64]),
    (50, [300, 5000, 20, 7, 90000, 1], [0, 50, 0, 50, 10, 40, 0]),
    (33, [40000, 40000, 40000, 40000], [0, 33, 0, 33, 33]),
    (90, [100, 200, 60], [90, 40, 97, 0]),
    (90, [100, 200, 60], [-7, 50, 1 << 30, 3]),
    (90, [1 << 30, -5, 2 ** 31 - 1], [0, 3, 93, 94]),
]


@pytest.mark.parametrize("heads,kv", [(4, 4), (12, 12), (8, 1)])
@pytest.mark.parametrize("n_tokens,lens,starts", FALLING)
def test_starts_that_fall(host, n_tokens, lens, starts, heads, kv):
    case = Case(lens, starts, n_tokens)
    for split in (1, 0):
        assert host.host_attend(ctypes.byref(case.c), heads, kv, 128, None, split) == 0
        check(host, case, heads // kv, kv)


@pytest.mark.parametrize("n_tokens,lens,starts", FALLING)
def test_a_row_has_one_owner(host, n_tokens, lens, starts):
    case = Case(lens, starts, n_tokens)
    want = [-1] * n_tokens
    for i, (start, n, _) in enumerate(case.rows()):
        want[start:start + n] = [i] * n
    assert host.host_append(ctypes.byref(case.c), 4, 64, 0, 1) == 0
    assert read(host.host_owners, I32) == want


@pytest.mark.parametrize("n_tokens,lens,starts", FALLING)
def test_latent_rows(host, n_tokens, lens, starts):
    case = Case(lens, starts, n_tokens, sum_len=sum(max(n, 0) for n in lens) % (1 << 22))
    assert host.host_latent(ctypes.byref(case.c), 5, 64, 256, 1) == 0
    check(host, case, 5, 1)


@pytest.mark.parametrize("seed", range(40))
def test_any_batch(host, seed):
    """Ordinary batches, and the same with starts in any order."""
    rng = random.Random(seed)
    n_seqs = rng.choice([1, 2, 5, 17, 64, 65, 130])
    news = [rng.choice([0, 1, 1, 2, rng.randint(1, 90)]) for _ in range(n_seqs)]
    lens = [n + rng.choice([0, 5, rng.randint(0, 400), rng.randint(0, 60000)]) for n in news]
    starts = [rng.randint(0, 3)]
    for n in news:
        starts.append(starts[-1] + n)
    n_tokens = max(starts[-1] + rng.randint(0, 3), 1)
    kv = rng.choice([1, 2, 4, 12])
    group = rng.choice([1, 2, 3, 4])
    if seed % 2:
        rng.shuffle(starts)
    case = Case(lens, starts, n_tokens, max_new=rng.choice([None, 1, 9, 64]), sum_len=rng.choice([0, sum(lens)]))
    spans = (Span * kv)(*[Span(rng.randint(0, 50), rng.choice([-1, rng.randint(0, 3000)])) for _ in range(kv)])
    assert host.host_attend(ctypes.byref(case.c), kv * group, kv, 64, rng.choice([None, spans]), 1) == 0
    check(host, case, group, kv)


@pytest.mark.parametrize("form,sum_len,tiles,hi", [(0, 0, 0, 2 ** 31 - 1), (0, 1100, 256, 63), (1, 1100, 0, 2 ** 31 - 1), (1, 0, 0, 2 ** 31 - 1)])
def test_form(host, form, sum_len, tiles, hi):
    """The form that is chosen expands a sequence's tokens only where their number is known."""
    case = Case([900, 200], [0, 200, 201], 201, sum_len=sum_len)
    assert host.host_latent(ctypes.byref(case.c), 3, 64, 256, form) == 0
    p = host.host_plan().contents
    assert (p.tiles, p.lo, p.hi) == (tiles, 1, hi)
    check(host, case, 3, 1)


@pytest.mark.parametrize("lens,pages,page,sum_len", [
    ([300, 0, 256, 257, 1, 5000] * 30, 512, 16, 30 * 6000), ([300, 5, 0, 700], 512, 16, 100),
    ([1 << 30] * 1024, 1024, 1 << 20, 1000),               # 2^40 tokens where 1000 are said to be
    ([2 ** 31 - 1, 5, -3] * 300, 1024, 1 << 20, 1 << 20)])
def test_rows_of_expanded_copies(host, lens, pages, page, sum_len):
    """Sequences follow one another in whole blocks, those beyond the room of the copies behind it."""
    case = Case(lens, list(range(len(lens) + 1)), len(lens), sum_len=sum_len, pages=pages, page=page)
    assert host.host_latent(ctypes.byref(case.c), 2, 64, 256, 2) == 0
    blocks = [-(-min(max(n, 0), pages * page) // 256) for n in lens]
    assert read(host.host_first_rows, ctypes.c_int64) == [256 * sum(blocks[:i]) for i in range(len(lens))]
    owned, room = [], -(-sum_len // 256) + len(lens)
    for i, n in enumerate(blocks):
        owned += [v for k in range(min(n, room - len(owned) // 2)) for v in (i, 256 * k)]
    assert read(host.host_blocks, I32, 2) == owned + [-1, -1] * (room - len(owned) // 2)


@pytest.mark.parametrize("heads,d,dtype", [(1, 8, 0), (12, 128, 0), (64, 64, 0), (64, 128, 0), (12, 128, 1), (64, 4096, 1), (3, 8192, 0)])
@pytest.mark.parametrize("n_tokens", [1, 7, 4680, (1 << 23) - 1, (1 << 23) + 1, 1 << 24])
def test_append_launches(host, heads, d, dtype, n_tokens):
    """Workgroups of 256 threads for at most 64 tokens each, fewer than 2^32 threads in all, whatever the rows' width."""
    case = Case([1], [0, 1], n_tokens)
    assert host.host_append(ctypes.byref(case.c), heads, d, dtype, 0) == 0
    tokens = host.host_block_tokens()
    assert 1 <= tokens <= 64 and -(-n_tokens // tokens) * 256 < 1 << 32


def overlapping(heads, tokens, width, head, token):
    rows = sorted(h * head + t * token for h in range(heads) for t in range(tokens))
    return any(b - a < width for a, b in zip(rows, rows[1:]))


@pytest.mark.parametrize("seed", range(6))
def test_outputs_that_overlap(seed):
    """Rows of an output that share elements are refused, whatever the strides of heads and tokens; others are not (that
    call then stops at its workspace)."""
    import paper_2605_09681_amd as fkv
    if not os.path.exists(fkv.LIB_PATH):
        build.build()
    rng = random.Random(seed)
    seen = set()
    cases = [(4, 6, 128, 128), (4, 6, 768, 128), (4, 6, 128, 512), (2, 3, 384, 256), (2, 50, 128, 256), (3, 2, 256, 384)]
    for k in range(400):
        heads, tokens = rng.choice([1, 2, 3, 5, 64]), rng.choice([1, 2, 3, 7, 40])
        head, token = (8 * rng.choice([0, 16, rng.randint(1, 40), rng.randint(1, 800), 16 * rng.randint(1, 100)]) for _ in range(2))
        cases.append((heads, tokens, head, token))
    for heads, tokens, head, token in cases:
        batch = fkv.fkv_batch(n_seqs=1, max_pages=4, page_tokens=16, n_pages=9, n_tokens=tokens, max_new=4, sum_len=70,
                              page_table=0x1000, seq_len=0x1000, q_start=0x1000)
        rows = lambda h, t: ctypes.byref(fkv.fkv_rows(0x1000, h, t))  # noqa: E731
        st = fkv.lib().fkv_latent_attention(ctypes.byref(batch), heads, 128, 256, rows(192, 12288), 0x1000, 0x1000, 0x1000, 1, None, 0.1,
                                            rows(head, token), 0, None, 0, None)
        assert st == 1
        bad = overlapping(heads, tokens, 128, head, token)
        assert ("overlap" in fkv.fkv_last_error()) == bad, (heads, tokens, head, token, fkv.fkv_last_error())
        seen.add(bad)
    assert seen == {True, False}
