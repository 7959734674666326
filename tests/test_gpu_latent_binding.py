"""What the tensor binding of the latent cache's and the pages' entry points refuses and returns:
arguments, gradients, versions of written tensors, streams, captured calls."""
import pytest

from tests.latent_problem import LatentProblem, PromptProblem
from tests.test_gpu_kv_cache import _randn
from tests.test_gpu_kv_streams import Pending, _ways

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


class Calls:
    """Every entry point on small inputs, with arguments that may be changed."""

    def __init__(self, kvr):
        import torch
        i32 = dict(dtype=torch.int32, device="cuda")
        self.kvr = kvr
        self.cache = kvr.LatentCache.allocate(kvr.KVR_KV_BF16, 4, 16, 256, 32)
        self.latent, self.key = _randn(1, (5, 256), "bf16"), _randn(2, (5, 32), "bf16")
        self.slots, self.pos = torch.arange(5, device="cuda"), torch.arange(5, **i32)
        self.table, self.w = kvr.kvr_rotary_table(32, 8), _randn(3, (256,), "bf16")
        self.att = dict(q=_randn(4, (2, 4, 288), "bf16"), cu_q=torch.tensor([0, 2], **i32), kv_len=torch.tensor([5], **i32),
                        page_table=torch.zeros(1, 1, **i32), max_q=2, max_kv=5, scale=0.1)
        self.pro = dict(q=_randn(5, (6, 4, 96), "bf16"), k=_randn(6, (9, 2, 64), "bf16"), k_rot=_randn(7, (9, 32), "bf16"),
                        v=_randn(8, (9, 2, 64), "bf16"), cu_q=torch.tensor([0, 6], **i32), cu_k=torch.tensor([0, 9], **i32),
                        max_q=6, max_k=9)
        self.refs, self.pages, self.len = (torch.zeros(*s, **i32) for s in ((9,), (3, 4), (3,)))
        self.none, self.two = torch.full((3,), -1, **i32), torch.tensor([20, 0, 33], **i32)
        self.buffers = kvr.PageBuffers(self.cache)
        self.pairs = torch.tensor([[0, 1], [-1, -1]], **i32)

    def write(self, **k):
        a = dict(cache=self.cache, latent=self.latent, key=self.key, slots=self.slots, check=False)
        return self.kvr.kvr_latent_write(**{**a, **k})

    def read(self, **k):
        return self.kvr.kvr_latent_read(**{**dict(cache=self.cache, slots=self.slots, check=False), **k})

    def attend(self, **k):
        return self.kvr.kvr_latent_attention(**{**dict(cache=self.cache, check=False), **self.att, **k})

    def prompt(self, **k):
        return self.kvr.kvr_latent_prompt(**{**self.pro, "check": False, **k})

    def fork(self, **k):
        a = dict(refs=self.refs, page_table=self.pages, kv_len=self.len, parent=self.none, page_size=16, check=False)
        return self.kvr.kvr_pages_fork(**{**a, **k})

    def resize(self, **k):
        a = dict(refs=self.refs, page_table=self.pages, kv_len=self.len, new_len=self.two, page_size=16, check=False)
        return self.kvr.kvr_pages_resize(**{**a, **k})

    def compact(self, **k):
        a = dict(refs=self.refs, page_table=self.pages, kv_len=self.len, page_size=16, check=False)
        return self.kvr.kvr_pages_compact(**{**a, **k})

    def copy(self, **k):
        return self.kvr.kvr_pages_copy(**{**dict(buffers=self.buffers, pairs=self.pairs, check=False), **k})


def test_refusals(kvr):
    import torch
    c = Calls(kvr)
    x, q = c.latent, c.att["q"]
    byte = torch.zeros(10, dtype=torch.uint8, device="cuda")
    mask = torch.tensor([[1], [3]], device="cuda")
    p = c.pro
    for call, bads in (
            (c.write, [dict(latent=x[:4]), dict(latent=x[:, :128]), dict(latent=x.half()), dict(key=c.key[:, :16]), dict(key=c.key.cpu()),
                       dict(slots=c.slots.int()), dict(table=c.table), dict(positions=c.pos), dict(norm_weight=c.w[:128]),
                       dict(norm_weight=c.w.float()), dict(latent=x.int()), dict(latent=x[None]), dict(status=byte)]),
            (c.read, [dict(dtype=torch.float64), dict(slots=c.slots.int()), dict(out=x), dict(out=torch.zeros(5, 288, device="cuda", dtype=torch.int32)),
                      dict(out=torch.zeros(5, 288, device="cuda"), dtype=torch.bfloat16)]),
            (c.attend, [dict(q=q[..., :256]), dict(q=q.double()), dict(cu_q=c.att["cu_q"][:1]), dict(kv_len=c.att["kv_len"].long()),
                        dict(page_table=c.att["page_table"][0]), dict(tree_mask=mask[:1]), dict(tree_mask=mask.int()), dict(out=q),
                        dict(out=torch.zeros(2, 4, 256, device="cuda")), dict(workspace=mask), dict(max_kv=1 << 40)]),
            (c.prompt, [dict(q=p["q"][..., :64]), dict(q=p["q"].half()), dict(k_rot=p["k_rot"][:8]), dict(k_rot=p["k_rot"][:, :16]),
                        dict(v=p["v"][:, :1]), dict(v=p["v"][:8]), dict(cu_q=p["cu_q"].long()), dict(cu_k=p["cu_k"][:1]),
                        dict(out=p["q"]), dict(max_q=1 << 33), dict(cu_q=p["cu_q"][0])]),
            (c.fork, [dict(parent=c.none.long()), dict(parent=c.none[:2]), dict(page_table=c.pages[:2]), dict(refs=c.refs.long()),
                      dict(kv_len=c.len.cpu()), dict(page_table=c.pages.t())]),
            (c.resize, [dict(new_len=c.two[:1]), dict(copies=torch.zeros(2, 2, dtype=torch.int32, device="cuda")), dict(workspace=c.refs)]),
            (c.compact, [dict(max_moves=10), dict(max_moves=-1), dict(moves=torch.zeros(8, 2, dtype=torch.int32, device="cuda")),
                         dict(used=torch.zeros(2, dtype=torch.int32, device="cuda"))]),
            (c.copy, [dict(pairs=c.pairs.long()), dict(pairs=c.pairs[:, :1]), dict(pairs=c.pairs.t())])):
        for bad in bads:
            with pytest.raises(ValueError):
                call(**bad)
    for call, bads in ((c.write, [dict(latent=None), dict(eps="x"), dict(cache=3), dict(cache=kvr.KvCache.allocate(0, 1, 1, 16, 64))]),
                       (c.attend, [dict(scale=None), dict(max_q="2"), dict(q=3)]), (c.prompt, [dict(k=None), dict(scale="1")]),
                       (c.fork, [dict(page_size=None)]), (c.copy, [dict(buffers=3), dict(buffers=c.cache)])):
        for bad in bads:
            with pytest.raises((TypeError, AttributeError)):
                call(**bad)
    for call, bad, code in ((c.attend, dict(q=q.half()), kvr.KVR_E_LAYOUT), (c.attend, dict(max_q=0), kvr.KVR_E_SIZE),
                            (c.attend, dict(scale=float("nan")), kvr.KVR_E_GRID), (c.write, dict(norm_weight=c.w, eps=-1.0), kvr.KVR_E_GRID),
                            (c.prompt, dict(max_k=0), kvr.KVR_E_SIZE), (c.prompt, {k: v.float() for k, v in p.items() if k in ("q", "k", "k_rot", "v")}, kvr.KVR_E_LAYOUT),
                            (c.fork, dict(page_size=24), kvr.KVR_E_LAYOUT), (c.resize, dict(page_size=8), kvr.KVR_E_LAYOUT),
                            (c.compact, dict(page_size=1 << 16), kvr.KVR_E_LAYOUT),
                            (c.fork, dict(page_table=c.pages[:1].expand(3, -1)), kvr.KVR_E_LAYOUT)):
        with pytest.raises(kvr.KvrError) as e:
            call(**bad)
        assert e.value.code == code
    with pytest.raises(ValueError):
        kvr.LatentCache.allocate(kvr.KVR_KV_FP4, 4, 16, 256, 32)
    small = kvr.LatentCache.allocate(kvr.KVR_KV_BF16, 3, 16, 256, 32)
    with pytest.raises(ValueError, match="same number of pages"):
        kvr.PageBuffers([c.cache, small])


def test_results_and_empty_calls(kvr):
    import torch
    c = Calls(kvr)
    c.write(norm_weight=c.w, positions=c.pos, table=c.table)
    out = torch.empty(5, 288, dtype=torch.bfloat16, device="cuda")
    assert c.read(out=out) is out and torch.equal(out, c.read())
    first, lse = c.attend(want_lse=True)
    assert first.shape == (2, 4, 256) and lse.shape == (2, 4) and lse.dtype == torch.float32
    assert torch.equal(first, c.attend(out=torch.empty_like(first), workspace=torch.empty(0, dtype=torch.uint8, device="cuda")))
    mask = torch.tensor([[1], [3]], device="cuda")   # a chain
    assert torch.equal(first, c.attend(tree_mask=mask))
    got, lse = c.prompt(want_lse=True)
    assert got.shape == (6, 4, 64) and torch.equal(got, c.prompt(out=torch.empty_like(got)))
    copies = torch.empty(3, 2, dtype=torch.int32, device="cuda")
    assert c.resize(copies=copies) is copies and c.pages[0, :2].tolist() == [0, 1] and c.pages[2, :3].tolist() == [2, 3, 4]
    moves, used = c.compact(max_moves=3)
    assert moves.shape == (3, 2) and int(used) == 5 and bool((moves == -1).all())
    assert c.copy() is None
    none = torch.empty(0, 288, dtype=torch.bfloat16, device="cuda")
    c.write(latent=none[:, :256], key=none[:, 256:], slots=c.slots[:0])
    assert c.read(slots=c.slots[:0]).shape == (0, 288)
    assert c.attend(q=c.att["q"][:0], cu_q=c.att["cu_q"][:1] * 0, kv_len=c.att["kv_len"][:0], page_table=c.att["page_table"][:0]).shape == (0, 4, 256)
    assert c.prompt(q=c.pro["q"][:0], cu_q=c.pro["cu_q"] * 0).shape == (0, 4, 64)
    assert float(c.prompt(k=c.pro["k"][:0], k_rot=c.pro["k_rot"][:0], v=c.pro["v"][:0], cu_k=c.pro["cu_k"] * 0).abs().max()) == 0
    c.copy(pairs=c.pairs[:0])
    c.fork(page_table=c.pages[:0], kv_len=c.len[:0], parent=c.none[:0])
    c.resize(page_table=c.pages[:0], kv_len=c.len[:0], new_len=c.none[:0])


def test_lost_gradients_are_refused(kvr):
    import torch
    c = Calls(kvr)
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    p, q = c.pro, c.att["q"]
    calls = [lambda t: c.write(latent=t(c.latent)), lambda t: c.write(key=t(c.key)), lambda t: c.write(norm_weight=t(c.w)),
             lambda t: c.write(cache=kvr.LatentCache(t(c.cache.rows), 32)), lambda t: c.attend(q=t(q)),
             lambda t: c.write(positions=c.pos, table=t(c.table)),
             lambda t: c.read(out=t(torch.empty(5, 288, dtype=torch.bfloat16, device="cuda"))),
             lambda t: c.attend(out=t(torch.empty(2, 4, 256, dtype=torch.bfloat16, device="cuda"))),
             lambda t: c.copy(buffers=kvr.PageBuffers(kvr.LatentCache(t(c.cache.rows), 32)))]
    calls += [lambda t, n=n: c.prompt(**{n: t(p[n])}) for n in ("q", "k", "k_rot", "v")]
    for call in calls:
        call(lambda t: t.clone())
        with pytest.raises(ValueError, match="requires gradients"):
            call(leaf)
        with torch.no_grad():
            call(leaf)
        with torch.inference_mode():
            call(leaf)


def test_written_tensors_are_noticed(kvr):
    import torch
    c = Calls(kvr)
    quant = kvr.LatentCache.allocate(kvr.KVR_KV_FP8, 4, 16, 256, 32)
    out, got = torch.empty(2, 4, 256, dtype=torch.bfloat16, device="cuda"), torch.empty(6, 4, 64, dtype=torch.bfloat16, device="cuda")
    rows = torch.empty(5, 288, dtype=torch.bfloat16, device="cuda")
    copies = torch.empty(3, 2, dtype=torch.int32, device="cuda")
    pool = [c.refs, c.pages, c.len]
    for call, ts in ((c.write, [c.cache.rows]), (lambda: c.write(cache=quant), [quant.rows, quant.scale]),
                     (lambda: c.read(out=rows), [rows]), (lambda: c.attend(out=out), [out]), (lambda: c.prompt(out=got), [got]),
                     (c.fork, pool), (lambda: c.resize(copies=copies), pool + [copies]), (c.compact, pool), (c.copy, [c.cache.rows])):
        before = [t._version for t in ts]
        call()
        assert [t._version for t in ts] == [n + 1 for n in before]
    before = c.cache.rows._version
    c.attend()
    c.read()
    assert c.cache.rows._version == before


@pytest.mark.parametrize("way", range(3))
def test_read_on_another_stream(kvr, way):
    import torch
    kw = _ways(kvr)[way]
    cache = kvr.LatentCache.allocate(kvr.KVR_KV_FP8, 256, 64, 512, 64)
    x, slots = _randn(1, (16384, 576), "bf16"), torch.randperm(16384, device="cuda")
    kvr.kvr_latent_write(cache, x[:, :512], x[:, 512:], slots)
    want = kvr.kvr_latent_read(cache, slots)
    p = Pending([2 * x.numel()])
    got = kvr.kvr_latent_read(cache, slots, stream=p.side, **kw)
    p.check((got, want))


@pytest.mark.parametrize("way", range(3))
def test_attention_on_another_stream(kvr, way):
    kw = _ways(kvr)[way]
    p = LatentProblem(kvr, 71, "bf16", [2000] * 16, [40] * 16, 64, 512, 64, 64)
    want = p.call()
    pending = Pending([want[0].numel() * 2])
    got = p.call(stream=pending.side, **kw)
    pending.check((got[0], want[0]))
    import torch
    assert torch.equal(got[1], want[1])


@pytest.mark.parametrize("way", range(3))
def test_prompt_on_another_stream(kvr, way):
    import torch
    kw = _ways(kvr)[way]
    p = PromptProblem(72, "bf16", [2500, 1500], [2500, 1500], 16, 1, 128, 64)
    want = p.call(kvr)
    pending = Pending([want[0].numel() * 2])
    got = p.call(kvr, stream=pending.side, **kw)
    pending.check((got[0], want[0]))
    assert torch.equal(got[1], want[1])


def test_pages_on_another_stream(kvr):
    """Calls in order on a stream of the caller's, with what they allocate."""
    import torch
    i32 = dict(dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()

    def run(**kw):
        refs, table, length = torch.zeros(70000, **i32), torch.full((200, 400), -1, **i32), torch.zeros(200, **i32)
        new = torch.arange(200, **i32) * 31
        if kw:
            side.wait_stream(torch.cuda.current_stream())
        a = kvr.kvr_pages_resize(refs, table, length, new, 16, check=False, **kw)
        b = kvr.kvr_pages_resize(refs, table, length, new // 3, 16, check=False, **kw)
        m, n = kvr.kvr_pages_compact(refs, table, length, 16, check=False, **kw)
        if kw:
            torch.cuda.current_stream().wait_stream(side)
        return refs, table, length, a, b, m, n

    for x, y in zip(run(), run(stream=side)):
        assert torch.equal(x, y)


def test_captured_calls(kvr):
    """Attention with and without a workspace, a prompt in parts, writes and the pages' calls in one
    graph, replayed with eager work between: every replay gives the eager results."""
    import torch
    i32 = dict(dtype=torch.int32, device="cuda")
    p = LatentProblem(kvr, 73, "bf16", [3000, 50], [2, 1], 40, 512, 64, 64)
    few = LatentProblem(kvr, 74, "fp8", [90, 700], [1, 1], 16, 256, 32, 16)
    pr = PromptProblem(75, "fp16", [100], [4000], 2, 1, 64, 32)
    refs, table, length = torch.zeros(500, **i32), torch.full((4, 100), -1, **i32), torch.zeros(4, **i32)
    goal, zero, parent = torch.tensor([300, 700, 0, -1], **i32), torch.zeros(4, **i32), torch.tensor([-1, -1, 1, 0], **i32)
    buffers = kvr.PageBuffers(kvr.LatentCache(torch.randn(500, 16, 288, device="cuda").bfloat16(), 32))

    def work():
        p.kvr.kvr_latent_write(p.cache, p.rows[:, :512], p.rows[:, 512:], p.slots, check=False)
        a, b, c = p.call(check=False), few.call(check=False), pr.call(kvr, check=False)
        kvr.kvr_pages_resize(refs, table, length, zero, 16, check=False)
        kvr.kvr_pages_resize(refs, table, length, goal, 16, check=False)
        kvr.kvr_pages_fork(refs, table, length, parent, 16, check=False)
        d = kvr.kvr_pages_resize(refs, table, length, length + 20, 16, check=False)
        m, n = kvr.kvr_pages_compact(refs, table, length, 16, max_moves=40, check=False)
        kvr.kvr_pages_copy(buffers, d, check=False)
        return [*a, *b, *c, d, m, n, refs.clone(), table.clone(), length.clone(), buffers.caches[0].rows.clone()]

    want = work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for i in range(4):
        for x in got:
            x.zero_()
        p.cache.rows.zero_()
        eager = work() if i % 2 else want
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y, z in zip(got, want, eager):
            assert torch.equal(x, y) and torch.equal(z, y)


def test_two_graphs_that_share_a_workspace(kvr):
    """Replayed in turn on one stream, with eager calls on the same workspace between."""
    import torch
    p = LatentProblem(kvr, 81, "bf16", [3000, 700], [1, 3], 40, 512, 64, 64)
    s = LatentProblem(kvr, 82, "fp8", [9000], [1], 16, 512, 64, 16)
    x = PromptProblem(83, "bf16", [50], [5000], 4, 2, 128, 64)
    ws = torch.full((1 << 26,), 0xFF, dtype=torch.uint8, device="cuda")
    calls = [lambda: p.call(workspace=ws, check=False), lambda: (*s.call(workspace=ws, check=False), *x.call(kvr, workspace=ws, check=False))]
    want = [c() for c in calls]
    graphs, got = [], []
    for c in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(c())
    for i in range(3):
        for g, out, ref, other in zip(graphs, got, want, calls[::-1]):
            for t in out:
                t.zero_()
            ws.fill_(i)
            if i:
                other()
            g.replay()
            assert all(torch.equal(a, b) for a, b in zip(out, ref))


def test_calls_at_the_same_time(kvr):
    """On four streams, with workspaces of their own."""
    import torch
    p = [LatentProblem(kvr, 90 + i, f, [4000 + 500 * i] * 3, [2] * 3, h, r, 64, 64)
         for i, (f, h, r) in enumerate([("bf16", 8, 512), ("fp8", 40, 256), ("fp16", 70, 256), ("bf16", 30, 512)])]
    want = [x.call() for x in p]
    streams = [torch.cuda.Stream() for _ in p]
    torch.cuda.synchronize()
    got = [[x.call(stream=s, check=False) for _ in range(5)] for x, s in zip(p, streams)]
    torch.cuda.synchronize()
    for w, each in zip(want, got):
        for g in each:
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])
