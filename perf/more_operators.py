"""Timing cases of the paged cache of many sequences: its write, attention of new
tokens over it, and attention over a paged cache of latent rows.

A case is a dict of plain values; ``op`` says which entry point it calls:

* ``append``  ``fkv_append_paged``: the new tokens of every sequence of a batch
              into their places in the pages;
* ``attend``  ``fkv_paged_attention``: attention of every sequence's new tokens
              over its pages, key heads shared by groups of query heads;
* ``latent``  ``fkv_latent_attention``: the same over a cache that holds one row
              for each token and all heads, a latent vector and a rotated key,
              from which every head's keys and values follow by a product.

``seqs`` lists the sequences, "tokens in the cache, new ones included + new
tokens" each.  ``heads`` query heads of ``d`` channels share ``kv`` key heads;
pages hold ``page`` tokens.  ``causal``: a new token sees keys up to its own;
else it sees its whole sequence (a chunk's tokens see one another).  The first
``limited`` key heads see only the first ``sink`` tokens and the ``recent``
tokens before their own (before the chunk, where not causal).  ``R`` latent
channels.  ``spare`` rows of the batch lie behind its last sequence.  ``layout``
is "token" for views of [tokens][heads][d] tensors, "head" for [heads][tokens][d].
"""
import math

import torch

own = False

ROT = 64                                 # channels of the rotated key of a latent row
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, seqs, **kw):
    c = dict(op=op, seqs=seqs, dtype="bf16", heads=12, kv=12, d=128, page=64, causal=True, limited=0, sink=0, recent=-1,
             R=0, lse=False, spare=0, layout="token")
    if name:
        c["name"] = name
    c.update(kw)
    return c


def listed():
    ragged = "812+1,4093+1,97+1,2600+1,1+1,6421+1,1540+1,333+1,5000+1,2049+1,64+1,3900+1,715+1,7800+1,1200+1,450+1"
    return [
        # a finished 480P chunk of one stream into pages of a frame each
        _case("append-480p", "append", "9360+4680", page=1560),
        # one token each of 16 streams: launch and host time
        _case("append-tokens", "append", ragged, heads=16, kv=16, d=64, page=16),
        # an AR step's chunk over all 21 frames of its history at 480P: the largest
        _case("attend-480p", "attend", "37440+4680", page=1560, causal=False),
        # one query token of one stream over the same history
        _case("attend-one-480p", "attend", "32761+1", page=1560, lse=True),
        # a step of 16 streams that answer token by token, key heads shared by four query heads
        _case("attend-tokens", "attend", ragged, heads=16, kv=4),
        # prompts of very different lengths, pages that end inside a tile
        _case("attend-prompts", "attend", "2900+2900,61+61,3500+3500,1733+1733", heads=40, kv=8, page=48),
        # streams that answer beside streams that read on, half of the key heads with a sink and a recent window
        _case("attend-mixed", "attend", "812+1,4093+5,97+97,2600+1,1+1,6421+600,1540+1,333+17", heads=16, kv=8, d=64, page=16,
              limited=4, sink=33, recent=700, lse=True, spare=3, layout="head"),
        # one token each of 16 streams over a latent cache
        _case("latent-tokens", "latent", ragged, heads=40, kv=1, R=512),
        # one token of one stream over a long latent cache
        _case("latent-one-480p", "latent", "32761+1", kv=1, R=256, page=1560),
        # a 480P chunk over a third of the history: every head's keys and values are made first
        _case("latent-480p", "latent", "15600+4680", kv=1, R=512, page=1560, causal=False),
        # a few tokens of short sequences, small heads: latency
        _case("latent-few", "latent", "75+5,130+3,9+9", heads=5, kv=1, d=64, R=256, page=16),
    ]


def _seqs(c):
    return [tuple(int(v) for v in s.split("+")) for s in c["seqs"].split(",")]


def _pairs(c, length, new, limited):
    """Visible (new token, key) pairs of a sequence."""
    t = torch.arange(length - new, length)
    end = t + 1 if c["causal"] else torch.full_like(t, length)
    if not limited:
        return int(end.sum())
    low = ((t if c["causal"] else torch.full_like(t, length - new)) - c["recent"]).clamp(min=0)
    return int((end - (low - torch.minimum(low, torch.full_like(low, c["sink"])))).sum())


def _keys(c, length, new, limited):
    """Keys of a sequence that some new token sees."""
    if not limited:
        return length
    low = max(length - new - c["recent"], 0)
    return length - max(low - c["sink"], 0)


def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    seqs = _seqs(c)
    n = sum(s[1] for s in seqs)
    width = c["R"] + ROT if c["R"] else c["d"]
    if c["op"] == "append":
        return {"bytes": 2 * n * c["kv"] * width * e * (1 if c["R"] else 2), "flops": 0}
    if c["op"] == "attend":
        cuts = [True] * c["limited"] + [False] * (c["kv"] - c["limited"])
        keys = sum(_keys(c, *s, cut) for s in seqs for cut in cuts)
        pairs = sum(_pairs(c, *s, cut) for s in seqs for cut in cuts) * (c["heads"] // c["kv"])
        return {"bytes": (2 * keys + 2 * n * c["heads"]) * c["d"] * e, "flops": 4 * c["d"] * pairs}
    keys = sum(_keys(c, *s, bool(c["limited"])) for s in seqs)
    pairs = sum(_pairs(c, *s, bool(c["limited"])) for s in seqs)
    absorbed = 2 * (2 * c["R"] + ROT) * pairs + 4 * c["d"] * c["R"] * n
    expanded = 2 * (2 * c["d"] + ROT) * pairs + 4 * c["d"] * c["R"] * keys
    return {"bytes": (keys * width + n * c["heads"] * (2 * c["d"] + ROT) + 2 * c["heads"] * c["d"] * c["R"]) * e,
            "flops": c["heads"] * min(absorbed, expanded)}


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["append", "attend", "attend", "attend", "latent", "latent"])
        kind = rng.choice(["tokens", "few", "prompts", "chunk", "mixed"])
        n_seqs = 1 if kind == "chunk" else log_int(1, 48)
        seqs = []
        for _ in range(n_seqs):
            k = rng.choice(["tokens", "few", "prompts", "chunk"]) if kind == "mixed" else kind
            new = {"tokens": 1, "few": rng.randint(2, 40), "prompts": log_int(1, 4000), "chunk": log_int(100, 5000)}[k]
            seqs.append((new + (0 if k == "prompts" else log_int(1, 30000) - 1), new))
        latent = op == "latent" or (op == "append" and rng.random() < 0.3)
        kv = 1 if latent else rng.choice([1, 2, 4, 8, 12, rng.randint(1, 20)])
        heads = rng.randint(1, 48) if latent else kv * rng.choice([1, 1, 2, 3, 4, 8])
        if heads > 64:
            continue
        limited = rng.randint(1, kv) if op != "append" and rng.random() < 0.4 else 0
        c = _case(None, op, ",".join("%d+%d" % s for s in seqs), heads=heads, kv=kv, d=rng.choice([64, 128, 128]),
                  dtype=rng.choice(["bf16", "bf16", "f32"]) if op == "append" else "bf16",
                  page=rng.choice([16, 32, 64, 128, log_int(1, 2000)]), causal=rng.random() < 0.7, limited=limited,
                  sink=rng.choice([0, 1, 4, log_int(1, 500)]) if limited else 0, recent=log_int(1, 8000) - 1 if limited else -1,
                  R=rng.choice([256, 512]) if latent else 0, lse=op == "attend" and rng.random() < 0.5,
                  spare=rng.choice([0, 0, rng.randint(1, 9)]), layout=rng.choice(["token", "token", "head"]))
        w = work(c)
        rows = sum(s[0] for s in seqs) * kv * (c["R"] + ROT if latent else 2 * c["d"])
        if w["flops"] <= 4e11 and w["bytes"] <= 4e8 and rows <= 3e8 and sum(s[1] for s in seqs) <= 12000:
            return c


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, seqs, page = _DT[c["dtype"]], _seqs(c), c["page"]
    n = sum(s[1] for s in seqs) + c["spare"]
    width = c["R"] + ROT if c["R"] else c["d"]
    rand = lambda *size: torch.randn(size, generator=g, device="cuda")  # noqa: E731

    def rows(heads, w):                  # [heads][n][w], a view of [n][heads][w] for the token layout
        x = (rand(n, heads, w) if c["layout"] == "token" else rand(heads, n, w)).to(dt)
        return x.transpose(0, 1) if c["layout"] == "token" else x

    # pages of a pool that other sequences use too, in any order
    counts = [-(-s[0] // page) for s in seqs]
    n_pages = sum(counts) + 2
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((len(seqs), max(counts)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, k in enumerate(counts):
        table[i, :k] = order[at:at + k]
        at += k
    starts = [sum(s[1] for s in seqs[:i]) for i in range(len(seqs) + 1)]
    s = dict(c=c, table=table, n_tokens=n, starts=starts,
             seq_len=torch.tensor([x[0] for x in seqs], dtype=torch.int32, device="cuda"),
             q_start=torch.tensor(starts, dtype=torch.int32, device="cuda"))
    s["K"] = rand(n_pages, c["kv"], page, width).to(dt)
    s["V"] = None if c["R"] else rand(n_pages, c["kv"], page, width).to(dt)
    if c["op"] == "append":
        s["K_new"], s["V_new"] = rows(c["kv"], width), None if c["R"] else rows(c["kv"], width)
        return s
    s["Q"] = rows(c["heads"], c["d"] + ROT if c["R"] else c["d"])
    o = torch.zeros((n, c["heads"], c["d"]) if c["layout"] == "token" else (c["heads"], n, c["d"]), dtype=dt, device="cuda")
    s["O"] = o.transpose(0, 1) if c["layout"] == "token" else o
    s["lse"] = torch.zeros((c["heads"], n), device="cuda") if c["lse"] else None
    if c["R"]:
        s["W_k"], s["W_v"] = ((rand(c["heads"], c["d"], c["R"]) / math.sqrt(c["R"])).to(dt) for _ in range(2))
    return s


def _scale(c):
    return 1 / math.sqrt(c["d"] + ROT if c["R"] else c["d"])


# -------------------------------------------------------------- plain forms
def _places(s, i, first, last):
    """Pool page and row of tokens first .. last - 1 of sequence i."""
    t = torch.arange(first, last, device="cuda")
    return s["table"][i].long()[t // s["c"]["page"]], t % s["c"]["page"]


def _mask(c, length, new, limited):
    """[new][length]: which keys a new token sees."""
    p = torch.arange(length - new, length, device="cuda")[:, None]
    j = torch.arange(length, device="cuda")[None]
    seen = j <= p if c["causal"] else j < length
    if limited:
        low = (p if c["causal"] else length - new) - c["recent"]
        seen = seen & ((j < c["sink"]) | (j >= low))
    return seen.expand(new, length)


def _weighted(z, seen, v):
    """softmax of z over the keys that are seen, times v; and the log of the sum."""
    z = torch.where(seen, z, -math.inf)
    m = z.amax(1, keepdim=True)
    p = (z - m).exp()
    total = p.sum(1, keepdim=True)
    return p @ v / total, (m + total.log())[:, 0]


def _plain_append(s):
    for i, (length, new) in enumerate(_seqs(s["c"])):
        page, row = _places(s, i, length - new, length)
        a, b = s["starts"][i], s["starts"][i + 1]
        s["K"][page, :, row] = s["K_new"][:, a:b].transpose(0, 1)
        if s["V"] is not None:
            s["V"][page, :, row] = s["V_new"][:, a:b].transpose(0, 1)
    return [s["K"]] if s["V"] is None else [s["K"], s["V"]]


def _plain_attend(s):
    c = s["c"]
    group = c["heads"] // c["kv"]
    for i, (length, new) in enumerate(_seqs(c)):
        page, row = _places(s, i, 0, length)
        a, b = s["starts"][i], s["starts"][i + 1]
        masks = [_mask(c, length, new, cut) for cut in (False, True)]
        for h in range(c["heads"]):
            y = h // group
            k, v = s["K"][page, y, row].float(), s["V"][page, y, row].float()
            z = s["Q"][h, a:b].float() @ k.T.contiguous() * _scale(c)
            o, lse = _weighted(z, masks[y < c["limited"]], v)
            s["O"][h, a:b] = o.to(s["O"].dtype)
            if c["lse"]:
                s["lse"][h, a:b] = lse
    return [s["O"], s["lse"]] if c["lse"] else [s["O"]]


def _plain_latent(s):
    c = s["c"]
    for i, (length, new) in enumerate(_seqs(c)):
        page, row = _places(s, i, 0, length)
        a, b = s["starts"][i], s["starts"][i + 1]
        x = s["K"][page, 0, row].float()
        latent, rotated = x[:, :c["R"]].contiguous(), x[:, c["R"]:]
        seen = _mask(c, length, new, bool(c["limited"]))
        for h in range(c["heads"]):
            k = torch.cat([latent @ s["W_k"][h].float().T.contiguous(), rotated], 1)
            v = latent @ s["W_v"][h].float().T.contiguous()
            z = s["Q"][h, a:b].float() @ k.T.contiguous() * _scale(c)
            s["O"][h, a:b] = _weighted(z, seen, v)[0].to(s["O"].dtype)
    return [s["O"]]


def _call(s):
    """The calls that a program makes, with the batch and the workspace that it keeps from pass to pass."""
    import paper_2605_09681_amd as fkv
    c = s["c"]
    if "batch" not in s:
        seqs = _seqs(c)
        s["batch"] = fkv.PagedBatch(s["table"], s["seq_len"], s["q_start"], c["page"], s["n_tokens"],
                                    max_new=max(x[1] for x in seqs), sum_len=sum(x[0] for x in seqs))
        if c["op"] == "attend":
            n = fkv.fkv_paged_attention_workspace_size(s["batch"], c["heads"], c["kv"], c["d"])
        elif c["op"] == "latent":
            n = fkv.fkv_latent_attention_workspace_size(s["batch"], c["heads"], c["d"], c["R"])
        else:
            n = 0
        s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    if c["op"] == "append":
        fkv.fkv_append_paged(s["batch"], s["K_new"], s["V_new"], s["K"], s["V"])
        return [s["K"]] if s["V"] is None else [s["K"], s["V"]]
    spans = [(c["sink"], c["recent"])] * c["limited"] + [(0, -1)] * (c["kv"] - c["limited"]) if c["limited"] else None
    if c["op"] == "latent":
        fkv.fkv_latent_attention(s["batch"], s["Q"], s["K"], s["W_k"], s["W_v"], _scale(c), s["O"], causal=c["causal"],
                                 span=spans and spans[0], workspace=s["ws"])
        return [s["O"]]
    fkv.fkv_paged_attention(s["batch"], s["Q"], s["K"], s["V"], _scale(c), s["O"], causal=c["causal"], spans=spans,
                            lse=s["lse"], workspace=s["ws"])
    return [s["O"], s["lse"]] if c["lse"] else [s["O"]]


def run(state):
    if own:
        return _call(state)
    return {"append": _plain_append, "attend": _plain_attend, "latent": _plain_latent}[state["c"]["op"]](state)


# --------------------------------------------------------------------- exact
def exact(case, seed):
    s = prepare(case, seed)
    c, page = s["c"], case["page"]
    seqs, table = _seqs(c), s["table"].tolist()
    if c["op"] == "append":
        out = []
        for pool, new in (("K", "K_new"), ("V", "V_new")):
            if s[pool] is None:
                continue
            out.append(s[pool].double())
            flat = out[-1].transpose(1, 2).reshape(-1, c["kv"], out[-1].shape[3])       # a copy: [pages * page][kv][width]
            row = s[new].double()
            for i, (length, n) in enumerate(seqs):
                at = [table[i][t // page] * page + t % page for t in range(length - n, length)]
                flat[torch.tensor(at, device="cuda")] = row[:, s["starts"][i]:s["starts"][i + 1]].transpose(0, 1)
            out[-1] = flat.reshape(out[-1].shape[0], page, c["kv"], -1).transpose(1, 2)
        return out
    O = torch.zeros(s["O"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(O.shape[:2], dtype=torch.float64, device="cuda")
    for i, (length, n) in enumerate(seqs):
        a, pos = s["starts"][i], torch.arange(length, device="cuda")
        own_pos = pos[length - n:]
        at = torch.tensor([table[i][t // page] * page + t % page for t in range(length)], device="cuda")
        for h in range(c["heads"]):
            y = 0 if c["R"] else h * c["kv"] // c["heads"]
            hidden = torch.zeros((n, length), dtype=torch.bool, device="cuda")
            if c["causal"]:
                hidden |= pos > own_pos[:, None]
            if y < c["limited"]:
                edge = own_pos[:, None] if c["causal"] else torch.full_like(own_pos[:, None], length - n)
                hidden |= (pos >= c["sink"]) & (pos < edge - c["recent"])
            q = s["Q"][h, a:a + n].double()
            x = s["K"][:, y].reshape(-1, s["K"].shape[3])[at].double()
            if c["R"]:                   # the products taken the other way round: by the query and by the output
                low, rot = x[:, :c["R"]].contiguous(), x[:, c["R"]:].contiguous()
                z = (q[:, :c["d"]] @ s["W_k"][h].double()) @ low.T.contiguous() + q[:, c["d"]:] @ rot.T.contiguous()
            else:
                z = q @ x.T.contiguous()
            z = (z * _scale(c)).masked_fill_(hidden, -math.inf)
            lse[h, a:a + n] = torch.logsumexp(z, 1)
            p = torch.softmax(z, 1)
            if c["R"]:
                O[h, a:a + n] = (p @ low) @ s["W_v"][h].double().T.contiguous()
            else:
                O[h, a:a + n] = p @ s["V"][:, y].reshape(-1, c["d"])[at].double()
    return [O, lse] if c["lse"] else [O]
