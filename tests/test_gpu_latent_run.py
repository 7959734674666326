"""The latent cache's and the pages' operators together, as a server of branching agents uses them:
rows in pages that are taken as they grow, branches that share and copy them, attention of all, the
pool brought together, everything given back.  And a prompt against the absorbed form of it."""
import math

import numpy as np
import pytest

from tests.latent_problem import check_rows, make_cache
from tests.test_gpu_kv_cache import _np, _randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


class Server:
    """Agents in two layers of one pool; every row of a cache is known by (agent's history, position)."""

    def __init__(self, kvr, fmt, pages, seqs, width, page, heads):
        import torch
        self.kvr, self.torch, self.page, self.fmt, self.heads = kvr, torch, page, fmt, heads
        self.dtype = "fp16" if fmt == "fp16" else "bf16"
        i32 = dict(dtype=torch.int32, device="cuda")
        self.refs, self.table = torch.zeros(pages, **i32), torch.full((seqs, width), -1, **i32)
        self.len = torch.zeros(seqs, **i32)
        self.layers = [make_cache(kvr, fmt, pages, page, 256, 64, fill=0xFF) for _ in range(2)]
        self.buffers = kvr.PageBuffers(self.layers)
        self.rope = kvr.kvr_rotary_table(64, 4096)
        self.weight = _randn(3, (256,), self.dtype)
        self.rows = [[{} for _ in range(seqs)] for _ in range(2)]   # layer, sequence: position -> row read back
        self.seed = 10

    def ints(self, x):
        return self.torch.tensor(x, dtype=self.torch.int32, device="cuda")

    def grow(self, new):
        """New lengths; what is new is written in both layers."""
        torch = self.torch
        old = self.len.tolist()
        pairs = self.kvr.kvr_pages_resize(self.refs, self.table, self.len, self.ints(new), self.page)
        self.kvr.kvr_pages_copy(self.buffers, pairs)
        seq, pos = [], []
        for b, (o, n) in enumerate(zip(old, new)):
            for layer in self.rows:
                for t in [t for t in layer[b] if 0 <= n <= t]:
                    del layer[b][t]
            seq += [b] * max(0, n - o)
            pos += range(o, max(o, n))
        if not seq:
            return
        s, t = torch.tensor(seq, device="cuda"), torch.tensor(pos, device="cuda")
        slots = self.table[s, t // self.page].long() * self.page + t % self.page
        for layer, cache in zip(self.rows, self.layers):
            self.seed += 1
            x = _randn(self.seed, (len(seq), 320), self.dtype)
            self.kvr.kvr_latent_write(cache, x[:, :256], x[:, 256:], slots, t.int(), self.rope, norm_weight=self.weight)
            for b, p, row in zip(seq, pos, _np(self.kvr.kvr_latent_read(cache, slots, torch.float32))):
                layer[b][p] = row

    def fork(self, parent):
        self.kvr.kvr_pages_fork(self.refs, self.table, self.len, self.ints(parent), self.page)
        for layer in self.rows:
            for b, a in enumerate(parent):
                if a >= 0:
                    layer[b] = dict(layer[a])

    def attend(self):
        """The newest token of each sequence that has one, in both layers, against its own history."""
        torch = self.torch
        lens = self.len.tolist()
        nq = [int(n > 0) for n in lens]
        cu = np.concatenate([[0], np.cumsum(nq)])
        outs = []
        for i, cache in enumerate(self.layers):
            q = _randn(100 + i, (int(cu[-1]), self.heads, 320), self.dtype)
            out, lse = self.kvr.kvr_latent_attention(cache, q, self.ints(cu), self.len, self.table, 1, max(lens), 0.06, want_lse=True)
            for b, n in enumerate(lens):
                if n:
                    x = np.stack([self.rows[i][b][t] for t in range(n)])
                    check_rows(_np(out[cu[b]]), _np(lse[cu[b]]), _np(q[cu[b]]), x, x[:, :256], np.ones((self.heads, n), bool), 0.06,
                               320, self.dtype, "fp16" if self.fmt == "fp16" else "bf16", (i, b))
            outs += [out, lse]
        return outs


@pytest.mark.parametrize("fmt,heads", [("bf16", 16), ("fp16", 40), ("fp8", 20)])
def test_branching_agents(kvr, fmt, heads):
    import torch
    s = Server(kvr, fmt, 60, 8, 12, 16, heads)
    s.grow([100, 37, 64, -1, -1, -1, -1, -1])
    s.attend()
    s.fork([-1, -1, -1, 0, 0, 1, 2, -1])
    s.attend()                                   # branches share every page
    s.grow([101, 40, -1, 105, 120, 38, 66, 5])   # and part, the parent too
    s.attend()
    s.grow([-1, 0, -1, 90, 0, -1, 65, -1])       # some end, some take tokens back
    s.grow([-1, -1, 70, 95, -1, 60, -1, -1])
    before = s.attend()
    moves, used = kvr.kvr_pages_compact(s.refs, s.table, s.len, 16)
    kvr.kvr_pages_copy(s.buffers, moves)
    held = s.table[torch.arange(12, device="cuda") < ((s.len + 15) // 16)[:, None]]
    assert int(held.max()) < int(used) == int((s.refs > 0).sum())
    for c in s.layers:                           # nothing beyond is needed any more
        c.rows[int(used):] = float("nan") if fmt != "fp8" else 0xFF
    for x, y in zip(before, s.attend()):
        assert torch.equal(x, y)
    s.grow([0] * 8)
    assert int(s.refs.abs().sum()) == 0


@pytest.mark.parametrize("past", [0, 300])
def test_prompt_and_absorbed_form_agree(kvr, past):
    """The same attention in both forms, each against the 64-bit definition from the same latents:
    keys and values expanded (rounded to 16 bits, as their product's result is), or the queries
    and outputs brought into the latent's space (rounded likewise)."""
    import torch
    heads, rank, rot, nope, n = 4, 256, 64, 128, 90
    total = past + n
    cache = make_cache(kvr, "bf16", total // 16 + 1, 16, rank, rot)
    x = _randn(1, (total, rank + rot), "bf16")
    slots = torch.arange(total, device="cuda")
    kvr.kvr_latent_write(cache, x[:, :rank], x[:, rank:], slots)
    wk, wv = (_randn(s, (heads, nope, rank), "bf16") * rank ** -0.5 for s in (2, 3))
    q = _randn(4, (n, heads, nope + rot), "bf16")
    scale = (nope + rot) ** -0.5
    i32 = dict(dtype=torch.int32, device="cuda")
    cu_q, lens = torch.tensor([0, n], **i32), torch.tensor([total], **i32)
    k, v = ((x[:, :rank] @ w.reshape(heads * nope, rank).t()).reshape(total, heads, nope) for w in (wk, wv))
    full = kvr.kvr_latent_prompt(q, k, x[:, rank:], v, cu_q, torch.tensor([0, total], **i32), n, total)
    absorbed = torch.cat([torch.stack([q[:, h, :nope] @ wk[h] for h in range(heads)], 1), q[..., nope:]], -1)
    pages = torch.arange(total // 16 + 1, **i32)[None]
    latent = kvr.kvr_latent_attention(cache, absorbed, cu_q, lens, pages, n, total, scale)
    mine = torch.stack([latent[:, h] @ wv[h].t() for h in range(heads)], 1)
    X, Q, K, V = _np(x), _np(q), _np(wk), _np(wv)
    seen = np.arange(total)[None] <= past + np.arange(n)[:, None]
    for h in range(heads):
        kk, vv = X[:, :rank] @ K[h].T, X[:, :rank] @ V[h].T
        s = scale * (Q[:, h, :nope] @ kk.T + Q[:, h, nope:] @ X[:, rank:].T)
        s = np.where(seen, s, -np.inf)
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        want = p @ vv
        # Scores: 16-bit keys are off by 2^-8 of each of nope products (times a few for their sum), and
        # so are absorbed queries in rank products: the sums of magnitudes bound both.
        eps = 2.0 ** -8
        ds = scale * np.maximum(np.abs(Q[:, h, :nope]) @ np.abs(kk).T, (np.abs(Q[:, h, :nope] @ K[h])) @ np.abs(X[:, :rank]).T)
        ds = 1.1 * eps * np.where(seen, ds, 0).max(1)
        # weights move by 2 ds and their own rounding, values, the latent's outputs and the results by
        # theirs: of |v| and, in the latent's space, of |x| |Wv|
        spread = p @ np.maximum(np.abs(vv), np.abs(X[:, :rank]) @ np.abs(V[h]).T)
        tol = (2 * ds[:, None] * np.exp(2 * ds[:, None]) + 4 * eps) * spread
        for got in (full, mine):
            assert (np.abs(_np(got[:, h]) - want) <= tol).all()
    assert math.isfinite(float(full.float().sum()))
