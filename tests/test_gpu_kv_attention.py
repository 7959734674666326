"""kvr_tree_attention against the plain 64-bit definition: formats, head layouts,
lengths, page sizes, masks, hidden non-finite values, streams and graphs."""
import math

import numpy as np
import pytest

from tests import kv_reference as ref
from tests.test_gpu_kv_cache import _cache, _dt, _np, _randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


def _tree(rng, n, words):
    """Ancestor masks of a random tree of n drafted tokens, [n, words] int64."""
    seen = []
    for i in range(n):
        parent = int(rng.integers(max(-1, i - 6), i))
        seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
    out = np.zeros((n, words), np.int64)
    for i, m in enumerate(seen):
        for w in range(words):
            x = (m >> (64 * w)) & (2 ** 64 - 1)
            out[i, w] = x - 2 ** 64 if x >> 63 else x
    return out


class Problem:
    """Sequences in a fragmented pool: unwritten rows hold 0xFF bytes (NaN in every
    format), the page table's unused entries -1."""

    def __init__(self, kvr, seed, fmt, dtype, kv, nq, heads, group, dim, page, tree=False, words=None,
                 order="hnd", table_slack=2, fill=0xFF, spread=1.0):
        import torch
        rng = self.rng = np.random.default_rng(seed)
        self.kvr, self.fmt, self.dtype, self.kv, self.nq = kvr, fmt, dtype, kv, nq
        self.heads, self.group, self.dim, self.page = heads, group, dim, page
        need = [-(-t // page) for t in kv]
        pages = sum(need) + 2
        self.cache = _cache(kvr, fmt, pages, heads, page, dim, order, fill=fill)
        ids = rng.permutation(pages)
        width = max(need + [1]) + table_slack
        table = np.full((len(kv), width), -1, np.int32)
        slots, at = [], 0
        for b, n in enumerate(need):
            table[b, :n] = ids[at:at + n]
            at += n
            t = np.arange(kv[b])
            slots.append(table[b, t // page].astype(np.int64) * page + t % page)
        self.first = np.concatenate([[0], np.cumsum(kv)])
        total = int(self.first[-1])
        self.slots = torch.from_numpy(np.concatenate(slots + [np.zeros(0, np.int64)])).cuda()
        self.k = _randn(seed + 1, (total, heads, dim), dtype, np.full((1, 1, 1), spread))
        self.v = _randn(seed + 2, (total, heads, dim), dtype)
        kvr.kvr_cache_write(self.cache, self.k, self.v, self.slots)
        self.table = torch.from_numpy(table).cuda()
        self.cu = np.concatenate([[0], np.cumsum(nq)])
        self.cu_q = torch.from_numpy(self.cu).int().cuda()
        self.kv_len = torch.tensor(kv, dtype=torch.int32, device="cuda")
        n = int(self.cu[-1])
        self.q = _randn(seed + 3, (n, heads * group, dim), dtype)
        self.max_q, self.max_kv = max(nq + [1]), max(kv + [1])
        self.words = words or -(-self.max_q // 64)
        self.mask = None
        if tree:
            self.mask = torch.from_numpy(np.concatenate(
                [_tree(rng, x, self.words) for x in nq] + [np.zeros((0, self.words), np.int64)])).cuda()
        self.scale = 1 / math.sqrt(dim)

    def call(self, **kw):
        args = dict(tree_mask=self.mask, scale=self.scale, want_lse=True)
        args.update(kw)
        return self.kvr.kvr_tree_attention(self.cache, self.q, self.cu_q, self.kv_len, self.table,
                                           self.max_q, self.max_kv, **args)

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

    def check(self, out, lse, rows=None):
        """Every output within the bound that the roundings give, derived below."""
        import torch
        k, v = (_np(x) for x in self.kvr.kvr_cache_read(self.cache, self.slots, torch.float32))
        q, out, lse = _np(self.q), _np(out), _np(lse)
        eps_o = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -11
        # the weights' type: the cache's, bfloat16 for the quantised ones
        eps_p, sub = (2.0 ** -11, 2.0 ** -25) if self.fmt == "fp16" else (2.0 ** -8, 0.0)
        for b, (t, n) in enumerate(zip(self.kv, self.nq)):
            if not n:
                continue
            seen = self.seen(b)
            for h in range(self.heads):
                kk, vv = (x[self.first[b]:self.first[b + 1], h] for x in (k, v))
                for gq in range(self.group):
                    head = h * self.group + gq
                    pick = np.arange(n) if rows is None or n <= rows else np.unique(
                        np.concatenate([[0, n - 1], self.rng.integers(0, n, rows)]))
                    qq = q[self.cu[b]:self.cu[b + 1], head][pick]
                    o, l, slack, spread = ref.attention(qq, kk, vv, seen[pick], self.scale)
                    # a score: dim + 8 roundings in 32 bits of at most `spread`; a weight twice
                    # that, its own rounding, the exponential's and the sums' (t terms)
                    ds = (self.dim + 16) * 2.0 ** -24 * spread
                    dw = eps_p + 2 * ds + (t + 64) * 2.0 ** -24 + 2.0 ** -21
                    vis = np.where(seen[pick][:, :, None], np.nan_to_num(np.abs(vv), posinf=0)[None], 0)
                    tol = dw[:, None] * slack * (1 + eps_o) + eps_o * np.abs(o) * 1.001 + sub * vis.sum(1) \
                        + (2.0 ** -25 if self.dtype == "fp16" else 0)
                    got = out[self.cu[b]:self.cu[b + 1], head][pick]
                    fine = np.isfinite(o)
                    assert np.array_equal(np.isfinite(got), fine), (b, head)
                    assert np.array_equal(np.isnan(got), np.isnan(o)), (b, head)
                    assert np.array_equal(got[np.isinf(o)], o[np.isinf(o)])
                    off = np.abs(got - o)[fine] - tol[fine]
                    assert (off <= 0).all(), (b, head, float(off.max()))
                    gl = lse[self.cu[b]:self.cu[b + 1], head][pick]
                    lt = ds + (t + 64) * 2.0 ** -24 + 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(l), l, 0)))
                    ok = np.isfinite(l)
                    assert np.array_equal(gl[~ok & ~np.isnan(l)], l[~ok & ~np.isnan(l)])
                    assert (np.abs(gl[ok] - l[ok]) <= lt[ok]).all(), (b, head)


LAYOUTS = [  # heads, group, dim, page
    (1, 1, 64, 16), (8, 4, 128, 16), (2, 8, 96, 32), (3, 3, 192, 64), (2, 1, 256, 256), (1, 40, 128, 32),
    (4, 16, 64, 64), (1, 7, 256, 16),
]


@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda x: "x".join(map(str, x)))
@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("fp16", "fp16"), ("fp8", "bf16"),
                                       ("fp8", "fp16"), ("fp4", "bf16"), ("fp4", "fp16")])
def test_decode(kvr, fmt, dtype, layout):
    """One new token of sequences from one cached token on, lengths around the tiles."""
    heads, group, dim, page = layout
    p = Problem(kvr, 21, fmt, dtype, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 128, 129, 517],
                [1] * 15, heads, group, dim, page, order="nhd" if heads == 2 else "hnd")
    p.check(*p.call())


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda x: "x".join(map(str, x)))
@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("fp16", "fp16"), ("fp8", "bf16"), ("fp4", "fp16")])
def test_drafts(kvr, fmt, dtype, layout, tree):
    """Runs and trees of up to 70 new tokens, sequences without any, and ones that are new
    from their first token on."""
    heads, group, dim, page = layout
    p = Problem(kvr, 22, fmt, dtype, [70, 5, 0, 40, 33, 300, 64, 1], [70, 5, 0, 0, 2, 37, 64, 1], heads,
                group, dim, page, tree=tree)
    p.check(*p.call(), rows=12)


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("nq", [1, 9])
def test_long_sequences_are_cut_and_joined(kvr, fmt, nq):
    p = Problem(kvr, 23, fmt, "bf16", [20011, 700, 9000], [nq, nq, 0], 2, 4, 128, 64, tree=nq > 1)
    p.check(*p.call(), rows=3)
    first = p.call()
    again = p.call()
    import torch
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_many_sequences(kvr):
    """More sequences than a wave has lanes, of very different lengths."""
    rng = np.random.default_rng(4)
    kv = [int(x) for x in np.exp(rng.uniform(0, math.log(1500), 150))]
    p = Problem(kvr, 24, "fp8", "bf16", kv, [min(t, int(rng.integers(0, 4))) for t in kv], 1, 2, 64, 16)
    p.check(*p.call())


@pytest.mark.parametrize("fmt", ["bf16", "fp16", "fp8"])
def test_empty_rows_and_any_mask(kvr, fmt):
    """Masks that leave rows empty (nothing cached before the drafts), hide a token from
    itself, and show later ones."""
    import torch
    dtype = fmt if fmt != "fp8" else "bf16"
    p = Problem(kvr, 25, fmt, dtype, [40, 12, 130], [40, 3, 30], 2, 3, 64, 16, tree=True)
    m = torch.from_numpy(np.random.default_rng(1).integers(-2 ** 62, 2 ** 62, p.mask.shape)).cuda()
    m[::3] = 0
    p.mask = m
    out, lse = p.call()
    p.check(out, lse)
    assert float(out[0].abs().max()) == 0 and bool((lse[0] == -math.inf).all())


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("fp16", "fp16"), ("fp8", "bf16"), ("fp4", "fp16")])
def test_hidden_tokens_may_hold_anything(kvr, fmt, dtype):
    """Infinities and NaN in drafted tokens that some rows do not see, in the rows past the
    end of the last page, and in pages that are not in use."""
    import torch
    p = Problem(kvr, 26, fmt, dtype, [90, 37], [20, 37], 2, 4, 128, 16, tree=True)
    base = int(p.first[1])
    for x, t, value in ((p.k, 75, math.inf), (p.v, 72, math.nan), (p.v, 80, math.inf), (p.v, 80 + 3, -math.inf),
                        (p.v, base + 9, math.nan), (p.v, base + 20, -math.inf), (p.k, base + 30, math.nan)):
        x[t, 1, 5] = value
    p.kvr.kvr_cache_write(p.cache, p.k, p.v, p.slots)
    out, lse = p.call()
    p.check(out, lse)
    assert bool(torch.isnan(out).any()) and bool(torch.isfinite(out).any(-1).any())


def test_large_scores(kvr):
    """Scores of several hundred: the running maximum moves by much, weights underflow."""
    p = Problem(kvr, 27, "bf16", "bf16", [700, 65], [3, 1], 2, 4, 128, 16, spread=60.0)
    p.check(*p.call())
    p.scale = -p.scale
    p.check(*p.call())
    p.scale = 0.0
    p.check(*p.call())


def test_strides_outputs_and_workspace(kvr):
    """q as part of a projection, out as a view, a workspace of the caller, no lse."""
    import torch
    p = Problem(kvr, 28, "fp8", "bf16", [9000, 37], [2, 1], 2, 4, 128, 32)
    want, _ = p.call()
    n, h = p.q.shape[:2]
    wide = torch.zeros((n, h + 4, 128), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:h + 2] = p.q
    p.q = wide[:, 2:h + 2]
    big = torch.full((h, n, 136), 9.0, dtype=torch.bfloat16, device="cuda")
    out = big.transpose(0, 1)[..., :128]
    ws = torch.full((1 << 24,), 171, dtype=torch.uint8, device="cuda")
    got = p.call(out=out, workspace=ws, want_lse=False)
    assert got.data_ptr() == out.data_ptr() and torch.equal(got, want)
    assert float((big[..., 128:] - 9).abs().max()) == 0


def test_domain_errors(kvr):
    import torch
    p = Problem(kvr, 29, "bf16", "bf16", [50, 33, 20], [2, 1, 1], 2, 2, 64, 16)
    want, _ = p.call()

    def fails(**kw):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.zeros_like(p.q)
        p.call(status=status, check=False, out=out, **kw)
        torch.cuda.synchronize()
        assert int(status.item()) == kvr.KVR_E_DOMAIN
        return out

    with pytest.raises(kvr.KvrError):
        p.table[1, 0] = p.cache.n_pages
        p.call()
    p.table[1, 0] = -5
    out = fails()
    assert torch.equal(out[:2], want[:2]) and torch.equal(out[3:], want[3:])
    for lens in ([1, 33, 20], [50, 10 ** 6, 20], [50, -3, 20], [50, 33 + 16 * 8, 20]):
        p.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        out = fails()
        b = 0 if lens[0] == 1 else 1
        assert float(out[p.cu[b]:p.cu[b + 1]].abs().max()) == 0   # left out
        assert torch.equal(out[3:], want[3:])
    p.kv_len = torch.tensor(p.kv, dtype=torch.int32, device="cuda")
    for cu in ([0, 2, 1, 4], [0, 2, 3, 900], [-1, 2, 3, 4]):
        p.cu_q = torch.tensor(cu, dtype=torch.int32, device="cuda")
        fails()


def test_offsets_beyond_4_gib(kvr):
    """A sequence whose pages lie on both sides of 4 GiB in the pool."""
    import torch
    pages, page = 9 * 1024, 64
    k = torch.full((pages, 32, page, 256), 0xFF, dtype=torch.uint8, device="cuda")
    sc = torch.full((pages, 32, page, 8), 0xFF, dtype=torch.uint8, device="cuda")
    p = Problem(kvr, 30, "fp8", "bf16", [200], [2], 32, 1, 256, 64)
    ids = torch.tensor([8300, 1, pages - 1, 4096], dtype=torch.int32, device="cuda")
    old = p.table[0, :4].long()
    for mine, theirs in ((k, p.cache.k), (sc, p.cache.k_scale)):
        mine[ids.long()] = theirs[old]
    p.cache.v.copy_(p.cache.k)
    p.cache.v_scale.copy_(p.cache.k_scale)
    want = p.call()
    p.cache = kvr.KvCache(k, k, sc, sc)
    p.table[0, :4] = ids
    got = p.call()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_side_stream(kvr):
    import torch
    p = Problem(kvr, 31, "fp4", "bf16", [5000, 90, 17], [4, 1, 1], 2, 4, 128, 64)
    want = p.call()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = p.call(stream=side, check=False)
    junk = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(8)]
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    del junk


def test_graph_replays(kvr):
    """Rotate, write and attend captured once; every replay, with eager work in between,
    gives the eager result bit for bit."""
    import torch
    p = Problem(kvr, 32, "fp8", "bf16", [3000, 33], [1, 1], 2, 4, 128, 16)
    table = kvr.kvr_rotary_table(128, 4096)
    pos = (p.kv_len - 1).int()
    new = p.slots[torch.tensor([2999, 3032], device="cuda")]
    x = _randn(5, (2, 2, 128), "bf16")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    q, out = torch.empty_like(p.q), torch.empty_like(p.q)

    def step():
        kvr.kvr_rotary(p.q, pos, table, out=q, check=False)
        kvr.kvr_cache_write(p.cache, x, x, new, pos, table, check=False)
        kvr.kvr_tree_attention(p.cache, q, p.cu_q, p.kv_len, p.table, 1, 3000, out=out, workspace=ws,
                               check=False)

    step()
    torch.cuda.synchronize()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        q.fill_(-7)
        out.fill_(-7)
        ws.fill_(171)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
