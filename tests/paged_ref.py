"""Paged batches and their attention in 64 bits, from the definition (tests only)."""
import math

import torch

ROT = 64


class Paged:
    """Sequences (tokens in the cache, of which new) whose pages lie anywhere in a pool."""

    def __init__(self, seqs, page, kv, width, seed=0, spare=0, dtype=torch.bfloat16, extra_pages=2, values=True, before=0):
        g = torch.Generator().manual_seed(seed)
        self.seqs, self.page, self.kv, self.width = seqs, page, kv, width
        counts = [-(-s[0] // page) for s in seqs]
        self.n_pages = sum(counts) + extra_pages
        order = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((len(seqs), max(max(counts), 1) + 1), -1, dtype=torch.int32)
        at = 0
        for i, k in enumerate(counts):
            self.table[i, :k] = order[at:at + k].int()
            at += k
        self.starts = [before + sum(s[1] for s in seqs[:i]) for i in range(len(seqs) + 1)]
        self.n_tokens = self.starts[-1] + spare
        self.K = torch.randn((self.n_pages, kv, page, width), generator=g).to(dtype)
        self.V = torch.randn((self.n_pages, kv, page, width), generator=g).to(dtype) if values else None
        self.g = g

    def rows(self, heads, width, dtype=torch.bfloat16):
        return torch.randn((heads, self.n_tokens, width), generator=self.g).to(dtype)

    def place(self, i, t):
        return int(self.table[i, t // self.page]), t % self.page

    def of(self, pool, i, y):
        """Rows of sequence i, head y, in order."""
        n = self.seqs[i][0]
        t = torch.arange(n)
        return pool[self.table[i].long()[t // self.page], y, t % self.page]

    def batch(self, fkv, max_new=None, sum_len=None, device="cuda"):
        to = lambda v: torch.tensor(v, dtype=torch.int32, device=device)  # noqa: E731
        return fkv.PagedBatch(self.table.to(device), to([s[0] for s in self.seqs]), to(self.starts), self.page, self.n_tokens,
                              max([s[1] for s in self.seqs] + [1]) if max_new is None else max_new,
                              sum(s[0] for s in self.seqs) if sum_len is None else sum_len)


def mask(length, new, causal, span):
    p = torch.arange(length - new, length)[:, None]
    j = torch.arange(length)[None]
    seen = (j <= p if causal else j < length).expand(new, length)
    if span is not None and span[1] >= 0:
        low = (p if causal else torch.full_like(p, length - new)) - span[1]
        seen = seen & ((j < span[0]) | (j >= low))
    return seen


def weighted(z, seen, v):
    """Rows' outputs, log sums and sums of p |v| over the keys that each sees; no key: 0 and -inf.  Values that a
    row does not see take no part, whatever they are."""
    o = torch.zeros((z.shape[0], v.shape[1]), dtype=torch.float64)
    a, lse = o.clone(), torch.full((z.shape[0],), -math.inf, dtype=torch.float64)
    z = torch.where(seen, z, -math.inf)
    some = seen.any(1)
    if some.any():
        lse[some] = torch.logsumexp(z[some], 1)
        p = torch.exp(z[some] - lse[some][:, None])
        clean = torch.where(torch.isfinite(v), v, 0.0)
        o[some], a[some] = p @ clean, p @ clean.abs()
        for j in (~torch.isfinite(v)).any(1).nonzero()[:, 0].tolist():
            odd = torch.where(torch.isfinite(v[j]), 0.0, v[j])
            o[seen[:, j]] += odd
    return o, lse, a


def attend(x, Q, scale, causal=True, spans=None):
    """(O, lse, A, |q||k| sums' largest a row) [heads][n_tokens]; A the sums of p |v|."""
    heads, n, d = Q.shape
    O = torch.zeros((heads, n, d), dtype=torch.float64)
    A, lse, top = O.clone(), torch.zeros((heads, n), dtype=torch.float64), torch.zeros((heads, n), dtype=torch.float64)
    for i, (length, new) in enumerate(x.seqs):
        a = x.starts[i]
        for h in range(heads):
            y = h * x.kv // heads
            k, v, q = x.of(x.K, i, y).double(), x.of(x.V, i, y).double(), Q[h, a:a + new].double()
            seen = mask(length, new, causal, spans and spans[y])
            o, s, w = weighted(q @ k.T * scale, seen, v)
            O[h, a:a + new], lse[h, a:a + new], A[h, a:a + new] = o, s, w
            if length and new:
                top[h, a:a + new] = torch.where(seen, q.abs() @ torch.nan_to_num(k, 0.0, 0.0, 0.0).abs().T * scale, 0.0).amax(1)
    return O, lse, A, top


def attend_latent(x, Q, W_k, W_v, scale, causal=True, span=None):
    """O and the sums of p |v|, from every head's keys and values."""
    heads, n, R = Q.shape[0], Q.shape[1], W_k.shape[2]
    d = W_k.shape[1]
    O = torch.zeros((heads, n, d), dtype=torch.float64)
    A = O.clone()
    for i, (length, new) in enumerate(x.seqs):
        a, row = x.starts[i], x.of(x.K, i, 0).double()
        seen = mask(length, new, causal, span)
        for h in range(heads):
            k = torch.cat([row[:, :R] @ W_k[h].double().T, row[:, R:]], 1)
            v = row[:, :R] @ W_v[h].double().T
            O[h, a:a + new], _, A[h, a:a + new] = weighted(Q[h, a:a + new].double() @ k.T * scale, seen, v)
    return O, A


def close(out, O, A, top, d, n_keys):
    """Output rows of bf16 against 64 bits.  Half a step of bf16 (2^-8) for the output and for each probability
    (on the sum of p |v|); a score is a sum of d products in fp32, off by d + 2 roundings of its absolute sum at the
    most, which moves probability and normaliser; the sums over keys, the exponentials (2^-21) in fp32."""
    err = (d + 2) * 2.0 ** -24 * top
    rel = torch.expm1(4 * err) + 2.0 ** -20 + n_keys * 2.0 ** -24
    tol = 2.0 ** -8 * (A + O.abs()) * (1 + 2.0 ** -7) + rel[..., None] * A
    return bool(((out.double() - O).abs() <= tol + 1e-30).all())


def close_lse(out, lse, top, d, n_keys):
    err = (d + 2) * 2.0 ** -24 * top + 2.0 ** -20 + n_keys * 2.0 ** -24 + 2.0 ** -22 * torch.nan_to_num(lse, neginf=0.0).abs()
    return bool(torch.where(torch.isinf(lse), out.double() == lse, (out.double() - lse).abs() <= err).all())


def rel2(out, ref):
    return float((out.double() - ref).norm() / ref.norm().clamp(min=1e-30))
