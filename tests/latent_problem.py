"""Latent caches, prompts and what their attention gives in 64 bits, for the tests on a GPU."""
from __future__ import annotations

import math

import numpy as np

from tests import kv_reference as ref
from tests.test_gpu_kv_attention import _tree
from tests.test_gpu_kv_cache import _dt, _np, _randn

EPS = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # half a step


def make_cache(kvr, fmt, pages, page, rank, rot, fill=None, order="ptr", slack=0):
    """A latent cache; order "tpr": token by token of all pages; slack: bytes between rows (16)."""
    import torch
    dim = rank + rot

    def new(width, dtype, pad):
        shape = (pages, page) if order == "ptr" else (page, pages)
        t = torch.zeros(shape + (width + pad,), dtype=dtype, device="cuda")
        if fill is not None:
            t.view(torch.uint8).fill_(fill)
        t = t[..., :width]
        return t if order == "ptr" else t.transpose(0, 1)

    if fmt == "fp8":
        return kvr.LatentCache(new(dim, torch.uint8, slack), rot, new(dim // 32, torch.uint8, slack and 3))
    return kvr.LatentCache(new(dim, _dt(fmt), slack // 2), rot)


def check_rows(got, lse, q, k, v, seen, scale, dim, dtype, weights, ids):
    """Rows of attention within the bounds that the roundings give.  got [rows, dv], lse [rows],
    q [rows, dim], k, v [tokens, ...], seen [rows, tokens], all in 64 bits."""
    width, t = v.shape[1], k.shape[0]
    o, l, slack, spread = ref.attention(q, k, np.pad(v, ((0, 0), (0, q.shape[1] - width))), seen, scale)
    o, slack = o[:, :width], slack[:, :width]
    eps_o = EPS[dtype]
    eps_p, sub = (2.0 ** -11, 2.0 ** -25) if weights == "fp16" else (2.0 ** -8, 0.0)
    # a score: dim + 8 roundings in 32 bits of at most `spread`; a weight twice that, its own
    # rounding, the exponential's and the sums' (t terms)
    with np.errstate(invalid="ignore", over="ignore"):
        ds = (dim + 16) * 2.0 ** -24 * spread
        dw = eps_p + 2 * ds + (t + 64) * 2.0 ** -24 + 2.0 ** -21
        vis = np.where(seen[:, :, None], np.nan_to_num(np.abs(v), posinf=0)[None], 0).sum(1) if sub else 0
        tol = dw[:, None] * slack * (1 + eps_o) + eps_o * np.abs(o) * 1.001 + sub * vis + \
            (2.0 ** -25 if dtype == "fp16" else 0)
        fine = np.isfinite(o)
        assert np.array_equal(np.isfinite(got), fine), ids
        assert np.array_equal(np.isnan(got), np.isnan(o)), ids
        assert np.array_equal(got[np.isinf(o)], o[np.isinf(o)]), ids
        off = np.abs(got - o)[fine] - tol[fine]
        assert (off <= 0).all(), (ids, float(off.max()))
        lt = ds + (t + 64) * 2.0 ** -24 + 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(l), l, 0)))
        ok = np.isfinite(l)
        assert np.array_equal(lse[~ok & ~np.isnan(l)], l[~ok & ~np.isnan(l)]), ids
        assert (np.abs(lse[ok] - l[ok]) <= lt[ok]).all(), ids


class LatentProblem:
    """Sequences in a fragmented pool: unwritten rows hold 0xFF bytes (NaN in every format), the
    page table's unused entries -1."""

    def __init__(self, kvr, seed, fmt, kv, nq, heads, rank, rot, page, tree=False, words=None, order="ptr", slack=0,
                 fill=0xFF, table_slack=2):
        import torch
        rng = self.rng = np.random.default_rng(seed)
        self.kvr, self.fmt, self.kv, self.nq, self.heads, self.rank, self.rot = kvr, fmt, kv, nq, heads, rank, rot
        self.page, self.dim = page, rank + rot
        self.dtype = "fp16" if fmt == "fp16" else "bf16"
        need = [-(-t // page) for t in kv]
        pages = sum(need) + 2
        self.cache = make_cache(kvr, fmt, pages, page, rank, rot, fill, order, slack)
        ids = rng.permutation(pages)
        table = np.full((len(kv), max(need + [1]) + table_slack), -1, np.int32)
        slots, at = [], 0
        for b, n in enumerate(need):
            table[b, :n] = ids[at:at + n]
            at += n
            t = np.arange(kv[b])
            slots.append(table[b, t // page].astype(np.int64) * page + t % page)
        self.first = np.concatenate([[0], np.cumsum(kv)])
        self.slots = torch.from_numpy(np.concatenate(slots + [np.zeros(0, np.int64)])).cuda()
        self.rows = _randn(seed + 1, (int(self.first[-1]), self.dim), self.dtype)
        self.write()
        self.table = torch.from_numpy(table).cuda()
        self.cu = np.concatenate([[0], np.cumsum(nq)])
        self.cu_q = torch.from_numpy(self.cu).int().cuda()
        self.kv_len = torch.tensor(kv, dtype=torch.int32, device="cuda")
        self.q = _randn(seed + 3, (int(self.cu[-1]), heads, self.dim), self.dtype)
        self.max_q, self.max_kv = max(nq + [1]), max(kv + [1])
        self.words = words or -(-self.max_q // 64)
        self.mask = None
        if tree:
            self.mask = torch.from_numpy(np.concatenate(
                [_tree(rng, x, self.words) for x in nq] + [np.zeros((0, self.words), np.int64)])).cuda()
        self.scale = 1 / math.sqrt(self.dim)

    def write(self):
        self.kvr.kvr_latent_write(self.cache, self.rows[:, :self.rank], self.rows[:, self.rank:], self.slots)

    def call(self, **kw):
        args = dict(tree_mask=self.mask, want_lse=True)
        args.update(kw)
        return self.kvr.kvr_latent_attention(self.cache, self.q, self.cu_q, self.kv_len, self.table, self.max_q,
                                             self.max_kv, self.scale, **args)

    def seen(self, b):
        n, t = self.nq[b], self.kv[b]
        s = np.ones((n, t), bool)
        if self.mask is None:
            s[:, t - n:] = np.tril(np.ones((n, n), bool))
        else:
            m = self.mask[self.cu[b]:self.cu[b + 1]].cpu().numpy()
            j = np.arange(n)
            s[:, t - n:] = (m[:, j // 64] >> (j % 64)) & 1
        return s

    def check(self, out, lse, rows=40, skip=()):
        import torch
        x = _np(self.kvr.kvr_latent_read(self.cache, self.slots, torch.float32))
        q, out, lse = _np(self.q), _np(out), _np(lse)
        for b, (t, n) in enumerate(zip(self.kv, self.nq)):
            if not n or b in skip:
                continue
            seen, xx = self.seen(b), x[self.first[b]:self.first[b + 1]]
            at = np.arange(n * self.heads)   # rows: query, head
            if len(at) > rows:
                at = np.unique(np.concatenate([[0, len(at) - 1], self.rng.integers(0, len(at), rows)]))
            i, h = at // self.heads, at % self.heads
            own = slice(self.cu[b], self.cu[b + 1])
            check_rows(out[own][i, h], lse[own][i, h], q[own][i, h], xx, xx[:, :self.rank], seen[i], self.scale, self.dim,
                       self.dtype, "fp16" if self.fmt == "fp16" else "bf16", b)


class PromptProblem:
    def __init__(self, seed, dtype, nq, nk, heads, group, nope, rot, causal=True, packed=True, spread=1.0):
        import torch
        self.dtype, self.nq, self.nk, self.heads, self.group = dtype, nq, nk, heads, group
        self.nope, self.rot, self.causal = nope, rot, causal
        self.rng = np.random.default_rng(seed)
        self.cu, self.ck = (np.concatenate([[0], np.cumsum(x)]) for x in (nq, nk))
        tq, tk = int(self.cu[-1]), int(self.ck[-1])
        self.q = _randn(seed, (tq, heads * group, nope + rot), dtype, np.full((1, 1, 1), spread))
        if packed:   # views of one product's result
            x = _randn(seed + 1, (tk, heads, 2 * nope), dtype)
            self.k, self.v = x[..., :nope], x[..., nope:]
            self.k_rot = _randn(seed + 2, (tk, 512 + rot), dtype)[:, 512:]
        else:        # heads first
            self.k, self.v = (_randn(seed + s, (heads, tk, nope), dtype).transpose(0, 1) for s in (1, 2))
            self.k_rot = _randn(seed + 3, (tk, rot), dtype)
        self.cu_q, self.cu_k = (torch.from_numpy(x).int().cuda() for x in (self.cu, self.ck))
        self.max_q, self.max_k = max(nq + [1]), max(nk + [1])
        self.scale = (nope + rot) ** -0.5

    def call(self, kvr, **kw):
        args = dict(causal=self.causal, scale=self.scale, want_lse=True)
        args.update(kw)
        return kvr.kvr_latent_prompt(self.q, self.k, self.k_rot, self.v, self.cu_q, self.cu_k, self.max_q, self.max_k,
                                     **args)

    def check(self, out, lse, rows=40):
        q, k, r, v, out, lse = (_np(x) for x in (self.q, self.k, self.k_rot, self.v, out, lse))
        total = self.heads * self.group
        for b, (n, m) in enumerate(zip(self.nq, self.nk)):
            if not n:
                continue
            own = slice(self.ck[b], self.ck[b + 1])
            for h in range(total):
                at = np.arange(n)
                if n > rows // total + 3:
                    at = np.unique(np.concatenate([[0, n - 1], self.rng.integers(0, n, rows // total + 3)]))
                seen = np.arange(m)[None] <= (m - n + at)[:, None] if self.causal else np.ones((len(at), m), bool)
                kk = np.concatenate([k[own, h // self.group], r[own]], 1)
                i = self.cu[b] + at
                check_rows(out[i, h], lse[i, h], q[i, h], kk, v[own, h // self.group], seen, self.scale,
                           self.nope + self.rot, self.dtype, self.dtype, (b, h))
