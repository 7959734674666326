"""The pages of a cache against a plain model of them: branches, lengths, compaction and copies,
in random runs over one pool, and the calls that are refused or reported."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


class Model:
    """refs, table and lengths as lists, one row and one page after another."""

    def __init__(self, n_pages, n_seqs, width, page):
        self.refs = np.zeros(n_pages, np.int32)
        self.table = np.full((n_seqs, width), -1, np.int32)
        self.len = np.zeros(n_seqs, np.int32)
        self.page = page

    def held(self, n):
        return -(-int(n) // self.page)

    def fork(self, parent):
        bad = False
        old = self.len.copy()
        for b, a in enumerate(parent):
            if a < 0:
                continue
            if a >= len(parent) or a == b or parent[a] >= 0 or old[b] != 0:
                bad = True
                continue
            n = self.held(old[a])
            self.table[b, :n] = self.table[a, :n]
            self.len[b] = old[a]
            for page in self.table[a, :n]:
                self.refs[page] += 1
        return bad

    def resize(self, new):
        refs = self.refs.copy()    # as the call finds them
        free = [int(p) for p in np.flatnonzero(refs == 0)]
        room, asked, bad = len(free), 0, False
        copies = np.full((len(new), 2), -1, np.int32)
        for b, want in enumerate(new):
            have, old = self.held(self.len[b]), int(self.len[b])
            if want < 0:
                continue
            need = self.held(want)
            if need > self.table.shape[1]:
                bad = True
                continue
            if want <= old:
                for e in range(need, have):
                    self.refs[self.table[b, e]] -= 1
                    self.table[b, e] = -1
                self.len[b] = want
                continue
            shared = old % self.page != 0 and refs[self.table[b, have - 1]] > 1
            take = need - have + shared
            asked += take
            if take and asked > room:
                bad = True
                continue
            got = free[asked - take:asked]
            if shared:
                copies[b] = self.table[b, have - 1], got[0]
                self.refs[self.table[b, have - 1]] -= 1
            first = have - shared
            self.table[b, first:first + take] = got
            self.refs[got] = 1
            self.len[b] = want
        return copies, bad

    def compact(self, most):
        moves = np.full((most, 2), -1, np.int32)
        for k in range(most):
            used, holes = np.flatnonzero(self.refs > 0), np.flatnonzero(self.refs == 0)
            if not len(used) or not len(holes) or holes[0] > used[-1]:
                break
            a, b = used[-1], holes[0]
            moves[k] = a, b
            self.refs[b], self.refs[a] = self.refs[a], 0
            for row, n in zip(self.table, self.len):
                row[:self.held(n)][row[:self.held(n)] == a] = b
        return moves, int((self.refs > 0).sum())


class Both:
    """The model and the GPU side by side."""

    def __init__(self, kvr, *shape):
        import torch
        self.kvr, self.torch, self.m = kvr, torch, Model(*shape)
        self.refs, self.len = (torch.from_numpy(x.copy()).cuda() for x in (self.m.refs, self.m.len))
        wide = torch.full((shape[1], shape[2] + 3), -7, dtype=torch.int32, device="cuda")
        self.wide, self.table = wide, wide[:, 1:1 + shape[2]]
        self.table.copy_(torch.from_numpy(self.m.table))
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def ints(self, x):
        return self.torch.tensor(np.asarray(x), dtype=self.torch.int32, device="cuda")

    def call(self, f, *args, **kw):
        self.status.zero_()
        return f(self.refs, self.table, self.len, *args, status=self.status, check=False, **kw)

    def same(self, bad):
        assert int(self.status.item()) == (self.kvr.KVR_E_DOMAIN if bad else 0)
        assert np.array_equal(self.refs.cpu().numpy(), self.m.refs)
        assert np.array_equal(self.len.cpu().numpy(), self.m.len)
        for got, want, n in zip(self.table.cpu().numpy(), self.m.table, self.m.len):
            n = self.m.held(n)
            assert np.array_equal(got[:n], want[:n])
        assert bool((self.wide[:, 0] == -7).all()) and bool((self.wide[:, -2:] == -7).all())

    def fork(self, parent):
        self.call(self.kvr.kvr_pages_fork, self.ints(parent), self.m.page)
        self.same(self.m.fork(parent))

    def resize(self, new):
        got = self.call(self.kvr.kvr_pages_resize, self.ints(new), self.m.page)
        copies, bad = self.m.resize(new)
        assert np.array_equal(got.cpu().numpy(), copies)
        self.same(bad)
        return got

    def compact(self, most=None):
        got, used = self.call(self.kvr.kvr_pages_compact, self.m.page, max_moves=most)
        moves, n = self.m.compact(len(self.m.refs) if most is None else most)
        assert np.array_equal(got.cpu().numpy(), moves) and int(used.item()) == n
        self.same(False)
        return got


@pytest.mark.parametrize("shape", [(40, 6, 8, 16), (300, 20, 40, 32), (1, 2, 3, 16), (64, 1, 64, 16), (130, 300, 2, 64)],
                         ids=lambda s: "x".join(map(str, s)))
def test_random_runs(kvr, shape):
    rng = np.random.default_rng(sum(shape))
    n_pages, n_seqs, width, page = shape
    x = Both(kvr, *shape)
    for step in range(40):
        what = rng.integers(0, 6)
        if what == 0:
            parent = np.full(n_seqs, -1)
            for b in rng.integers(0, n_seqs, 1 + n_seqs // 3):
                parent[b] = rng.integers(-1, n_seqs + 1)
            x.fork(parent)
        elif what == 1:
            x.compact(None if rng.random() < 0.5 else int(rng.integers(0, n_pages + 1)))
        else:
            new = np.full(n_seqs, -1)
            some = rng.random(n_seqs) < 0.6
            near = x.m.len + rng.integers(-2 * page, 2 * page + 1, n_seqs)
            new[some] = np.where(rng.random(n_seqs) < 0.3, rng.integers(0, width * page + 2, n_seqs), near.clip(0))[some]
            x.resize(new)
    x.resize(np.zeros(n_seqs, int))
    assert x.m.refs.sum() == 0


def test_pools_of_several_chunks(kvr):
    """More pages than one block counts, rows of thousands of entries, holes far apart."""
    rng = np.random.default_rng(5)
    x = Both(kvr, 40000, 70, 3000, 16)
    x.resize(rng.integers(0, 8000, 70))
    x.resize(np.where(np.arange(70) % 3 == 0, 0, -1))
    x.fork(np.where(np.arange(70) % 3 == 0, (np.arange(70) + 1) % 70, -1))
    x.resize(np.where(np.arange(70) % 3 == 0, x.m.len + 700, -1))
    x.compact(500)
    x.compact()
    x.resize(np.full(70, 40000))        # more than there are
    x.resize(np.full(70, 3000 * 16 + 1))   # more than a row has room for
    x.resize(np.zeros(70, int))


def test_many_rows(kvr):
    rng = np.random.default_rng(6)
    x = Both(kvr, 9000, 2500, 4, 16)
    x.resize(rng.integers(0, 50, 2500))
    x.resize(x.m.len + rng.integers(0, 3, 2500))
    x.resize(np.where(rng.random(2500) < 0.5, 0, -1))
    x.compact()


def test_every_sharer_grows(kvr):
    """A shared partial page whose holders all grow at once is copied by each and then free."""
    x = Both(kvr, 30, 4, 5, 16)
    x.resize([20, 0, 0, 0])
    x.fork([-1, 0, 0, 0])
    copies = x.resize([30, 21, 40, 20])
    assert copies[:3, 0].tolist() == [1, 1, 1] and copies[3].tolist() == [-1, -1]
    x.resize([-1, -1, -1, 32])          # the last holder keeps it
    assert x.m.refs[1] == 1


def test_exact_fit_and_one_too_many(kvr):
    x = Both(kvr, 10, 3, 10, 16)
    x.resize([48, 48, 64])
    x.resize([-1, -1, 65])
    x.resize([40, -1, -1])              # shrinks within its last page
    x.resize([48, -1, -1])              # and grows back into it without a free one
    assert x.m.len.tolist() == [48, 48, 64]


def test_rows_that_do_not_fit(kvr):
    """Lengths and entries that are not the pool's are reported, and nothing outside is touched."""
    import torch
    refs, table, kv = (torch.zeros(*s, dtype=torch.int32, device="cuda") for s in ((20,), (3, 4), (3,)))
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731

    def fails(f, *args):
        with pytest.raises(kvr.KvrError) as e:
            f(refs, table, kv, *args)
        assert e.value.code == kvr.KVR_E_DOMAIN

    kv.copy_(ints(-5, 70, 0))           # below 0, and more entries than a row has
    fails(kvr.kvr_pages_resize, ints(3, 1, -1), 16)
    assert kv.tolist() == [-5, 70, 0] and int(refs.sum()) == 0
    fails(kvr.kvr_pages_fork, ints(-1, -1, 0), 16)
    fails(kvr.kvr_pages_fork, ints(-1, -1, 1), 16)
    fails(kvr.kvr_pages_compact, 16)
    kv.copy_(ints(20, 0, 0))
    table[0, :2] = ints(5, 20)          # a page outside
    refs[5] = 1
    fails(kvr.kvr_pages_fork, ints(-1, 0, -1), 16)
    fails(kvr.kvr_pages_resize, ints(25, -1, -1), 16)
    assert kv[0] == 20
    fails(kvr.kvr_pages_resize, ints(0, 0, -1), 16)
    assert int(refs.abs().sum()) <= 1
    kv.copy_(ints(10, 0, 0))
    refs.zero_()
    table[0, 0] = 3                     # given back more often than held
    fails(kvr.kvr_pages_resize, ints(0, -1, -1), 16)
    assert int(refs[3]) == 0


CACHES = [("bf16", 4, 16, 64), ("fp8", 2, 16, 96), ("fp4", 3, 32, 64), ("latent-fp16", 1, 16, 256), ("latent-fp8", 1, 64, 512)]


def _bytes(c):
    return [t for t in c.tensors if t is not None]


@pytest.mark.parametrize("order", ["hnd", "nhd", "pages inside"])
@pytest.mark.parametrize("kind", CACHES, ids=lambda c: c[0])
def test_copies(kvr, kind, order):
    """Every tensor of every layer, whatever its strides; nothing but the target pages changes."""
    import torch
    fmt, heads, page, dim = kind
    pages, gen = 50, torch.Generator("cuda").manual_seed(1)

    def rand(shape, dtype):
        if order == "nhd" and len(shape) == 4:
            t = rand_flat((shape[0], shape[2], shape[1], shape[3] + 16), dtype)[..., :shape[3]].transpose(1, 2)
        elif order == "pages inside":   # [.., pages, row]
            t = rand_flat(shape[1:-1] + (shape[0], shape[-1]), dtype).movedim(-2, 0)
        else:
            t = rand_flat(shape, dtype)
        return t

    def rand_flat(shape, dtype):
        n = torch.empty(0, dtype=dtype).element_size()
        raw = torch.randint(0, 256, shape[:-1] + (shape[-1] * n,), dtype=torch.uint8, generator=gen, device="cuda")
        return raw.view(dtype)

    def one():
        if fmt.startswith("latent"):
            if fmt.endswith("8"):
                return kvr.LatentCache(rand((pages, page, dim + 32), torch.uint8), 32, rand((pages, page, (dim + 32) // 32), torch.uint8))
            return kvr.LatentCache(rand((pages, page, dim + 32), torch.float16), 32)
        if fmt == "bf16":
            return kvr.KvCache(*(rand((pages, heads, page, dim), torch.bfloat16) for _ in "kv"))
        row = dim if fmt == "fp8" else dim // 2
        return kvr.KvCache(*(rand((pages, heads, page, n), torch.uint8) for n in (row, row, dim // 32, dim // 32)))

    caches = [one() for _ in range(3)]
    pairs = torch.tensor([[3, 7], [-1, 9], [49, 0], [3, 11], [5, -1], [-1, -1], [20, 48]], dtype=torch.int32, device="cuda")
    raw = lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    want = [raw(t).clone() for c in caches for t in _bytes(c)]
    for w in want:
        for a, b in ((3, 7), (49, 0), (3, 11), (20, 48)):
            w[b] = w[a]
    kvr.kvr_pages_copy(kvr.PageBuffers(caches), pairs)
    for w, t in zip(want, [t for c in caches for t in _bytes(c)]):
        assert torch.equal(w, raw(t))
    pairs[1, 0] = 50
    with pytest.raises(kvr.KvrError) as e:
        kvr.kvr_pages_copy(kvr.PageBuffers(caches), pairs)
    assert e.value.code == kvr.KVR_E_DOMAIN
    for w, t in zip(want, [t for c in caches for t in _bytes(c)]):
        assert torch.equal(w, raw(t))


def test_copies_of_many_layers_and_large_pages(kvr):
    import torch
    caches = [kvr.LatentCache(torch.randn(6, 256, 320, device="cuda").bfloat16(), 64) for _ in range(70)]
    caches.append(kvr.KvCache(*(torch.randn(6, 2, 16, 64, device="cuda").half() for _ in "kv")))
    before = [[t.clone() for t in _bytes(c)] for c in caches]
    pairs = torch.tensor([[0, 5], [1, 4]], dtype=torch.int32, device="cuda")
    buffers = kvr.PageBuffers(caches)
    for _ in range(2):
        kvr.kvr_pages_copy(buffers, pairs)
    for c, b in zip(caches, before):
        for t, w in zip(_bytes(c), b):
            w[5], w[4] = w[0], w[1]
            assert torch.equal(t, w)


def test_offsets_beyond_32_bits(kvr):
    import torch
    rows = torch.zeros((1 << 32) // (320 * 2 * 64) + 30, 64, 320, dtype=torch.float16, device="cuda")
    last = rows.shape[0] - 1
    rows[last] = 3
    kvr.kvr_pages_copy(kvr.PageBuffers(kvr.LatentCache(rows, 64)),
                       torch.tensor([[last, last - 1]], dtype=torch.int32, device="cuda"))
    assert float(rows[last - 1].min()) == 3 and float(rows[last - 2].max()) == 0


@pytest.mark.parametrize("shape", [(2048, 30, 90, 16), (2049, 30, 90, 16), (4096, 64, 80, 16), (4097, 20, 300, 16), (4096, 65, 80, 32),
                                   (2048, 1024, 4, 16), (2048, 1025, 4, 16), (2000, 40, 1639, 16)],
                         ids=lambda s: "x".join(map(str, s)))
def test_random_runs_of_larger_pools(kvr, shape):
    """Sizes about which the calls change from one launch to several."""
    rng = np.random.default_rng(sum(shape))
    n_pages, n_seqs, width, page = shape
    width = min(width, 2 * n_pages // n_seqs)   # of the lengths that are asked for
    x = Both(kvr, *shape)
    for step in range(6):
        new = rng.integers(0, width * page + 1, n_seqs)
        x.resize(np.where(rng.random(n_seqs) < 0.3, 0, np.where(rng.random(n_seqs) < 0.5, -1, new)))
        parent = np.where((x.m.len == 0) & (rng.random(n_seqs) < 0.8), rng.integers(0, n_seqs, n_seqs), -1)
        parent[parent == np.arange(n_seqs)] = -1
        x.fork(parent)
        x.resize(np.where(rng.random(n_seqs) < 0.5, x.m.len + rng.integers(0, 2 * page, n_seqs), -1))
        x.compact(None if step % 2 else 40)
    x.resize(np.zeros(n_seqs, int))
    assert x.m.refs.sum() == 0


@pytest.mark.parametrize("n_pages", [300, 2048, 3000, 40000])
def test_a_free_page_given_back_while_it_is_taken(kvr, n_pages):
    """A row that names free pages ends, and one that takes these pages grows in the same call: the
    first is reported, the second has them."""
    import torch
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    n = min(n_pages, 1500) - 5
    table = torch.full((4, n), -1, dtype=torch.int32, device="cuda")
    for _ in range(5):
        refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        refs[:3] = 2                              # of rows that are not in the table
        table[0] = torch.arange(n - 1, -1, -1, device="cuda") + 3
        table[2] = table[0]
        table[2, 0] = 1                           # a page that it does hold
        kv, copies = ints(16 * n, 0, 16 * n, 0), None
        for check in (False, True):               # the second call finds all in order
            status = ints(0)
            new = ints(0, 16 * n - 3, 0, -1)
            copies = kvr.kvr_pages_resize(refs, table, kv, new, 16, copies=copies, status=status, check=check)
            assert int(status.item()) == (0 if check else kvr.KVR_E_DOMAIN)
            assert kv.tolist() == [0, 16 * n - 3, 0, 0] and bool((copies == -1).all())
            assert refs[:3].tolist() == [2, 1, 2] and bool((refs[3:3 + n] == 1).all()) and not refs[3 + n:].any()
            assert torch.equal(table[1], torch.arange(n, device="cuda").int() + 3)
            assert bool((table[0] == -1).all()) and bool((table[2] == -1).all())


@pytest.mark.parametrize("n_pages", [5, 5000])
def test_copies_of_a_call_that_fails_for_another_row(kvr, n_pages):
    """Three rows share a page and grow, one of them too far: the error brings the copies of the
    others, whose pages have changed already."""
    import torch
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = kvr.LatentCache(torch.randn(n_pages, 16, 288, device="cuda").bfloat16(), 32)
    refs, table, kv = ints(*[0] * n_pages), torch.full((3, n_pages), -1, dtype=torch.int32, device="cuda"), ints(0, 0, 0)
    kvr.kvr_pages_resize(refs, table, kv, ints(20, 0, 0), 16)
    kvr.kvr_pages_fork(refs, table, kv, ints(-1, 0, 0), 16)
    with pytest.raises(kvr.KvrError) as e:
        kvr.kvr_pages_resize(refs, table, kv, ints(21, 22, 16 * n_pages), 16)
    assert e.value.code == kvr.KVR_E_DOMAIN
    assert e.value.copies.tolist() == [[1, 2], [1, 3], [-1, -1]] and kv.tolist() == [21, 22, 20]
    kvr.kvr_pages_copy(kvr.PageBuffers(cache), e.value.copies)
    assert torch.equal(cache.rows[2], cache.rows[1]) and torch.equal(cache.rows[3], cache.rows[1])
    kvr.kvr_pages_resize(refs, table, kv, ints(0, -1, -1), 16)   # a hole at 2
    kv[0] = -1
    with pytest.raises(kvr.KvrError) as e:
        kvr.kvr_pages_compact(refs, table, kv, 16, max_moves=2)
    assert e.value.moves.tolist() == [[3, 2], [-1, -1]] and e.value.used.tolist() == [3]
    assert table[1, :2].tolist() == [0, 2]
    with pytest.raises(kvr.KvrError) as e:   # refused on the host: nothing was done
        kvr.kvr_pages_resize(refs, table, kv, ints(0, -1, -1), 15)
    assert not hasattr(e.value, "copies")
