"""Calls on another stream than torch's current one: memory that a call allocates may have
been freed with work on it still queued, and neither that work nor the call may see the
other's values."""
import pytest

from tests.test_gpu_kv_attention import Problem
from tests.test_gpu_kv_bounds import _workspace_bytes
from tests.test_gpu_kv_cache import _randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


class Pending:
    """Blocks of memory that are freed while the current stream still has to read them, and
    then to write them."""

    def __init__(self, sizes):
        import torch
        self.torch = torch
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        a = torch.randn(4096, 4096, device="cuda").bfloat16()
        b = torch.empty_like(a)
        self.plugs = []   # in place of the free memory that the call might take instead
        for n in sorted(sizes):
            reserved = torch.cuda.memory_reserved()
            while torch.cuda.memory_reserved() == reserved:
                self.plugs.append(torch.empty(n, dtype=torch.uint8, device="cuda"))
        blocks = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda") for n in sizes]
        self.copies = [torch.zeros_like(x) for x in blocks]
        torch.cuda.synchronize()
        for _ in range(200):   # well beyond the time that the host takes to make the call
            torch.mm(a, a, out=b)
        for x, y in zip(blocks, self.copies):
            y.copy_(x)
            x.fill_(0xFF)
        self.at = [range(x.data_ptr(), x.data_ptr() + n) for x, n in zip(blocks, sizes)]
        self.side = torch.cuda.Stream()
        self.keep = a, b
        blocks.clear()
        del x, y

    def took(self, x):
        return any(x.data_ptr() in at for at in self.at)

    def check(self, *results):
        """After the call: what was queued has read its own values.  ``results``: tensors
        that should have taken the blocks, and what they should hold."""
        self.torch.cuda.synchronize()
        assert all(bool((y == 0x5A).all()) for y in self.copies)
        for got, want in results:
            assert self.took(got)   # else nothing was tested
            assert self.torch.equal(got, want)


def _ways(kvr):
    """Keywords: without waiting for the device, and with a status of the caller's."""
    import torch
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    return dict(check=False), dict(status=status, check=True), dict(status=status, check=False)


@pytest.mark.parametrize("way", range(3))
def test_rotary(kvr, way):
    import torch
    kw = _ways(kvr)[way]
    x = _randn(1, (4096, 16, 128), "bf16")
    pos = torch.arange(4096, device="cuda").int()
    table = kvr.kvr_rotary_table(128, 4096)
    want = kvr.kvr_rotary(x, pos, table)
    p = Pending([2 * x.numel()])
    got = kvr.kvr_rotary(x, pos, table, stream=p.side, **kw)
    p.check((got, want))


def test_rotary_table(kvr):
    want = kvr.kvr_rotary_table(128, 65536)
    p = Pending([4 * want.numel()])
    p.check((kvr.kvr_rotary_table(128, 65536, stream=p.side), want))


@pytest.mark.parametrize("way", range(3))
def test_read(kvr, way):
    import torch
    kw = _ways(kvr)[way]
    n, heads, dim = 8192, 8, 128
    cache = kvr.KvCache.allocate(kvr.KVR_KV_FP8, n // 64, heads, 64, dim)
    x, y = _randn(1, (n, heads, dim), "bf16"), _randn(2, (n, heads, dim), "bf16")
    slots = torch.randperm(n, device="cuda")
    kvr.kvr_cache_write(cache, x, y, slots)
    want = kvr.kvr_cache_read(cache, slots)
    p = Pending([2 * x.numel()] * 2)
    got = kvr.kvr_cache_read(cache, slots, stream=p.side, **kw)
    p.check(*zip(got, want))


@pytest.mark.parametrize("lse", [False, True])
@pytest.mark.parametrize("way", range(3))
def test_attention(kvr, way, lse):
    """The output, the workspace of sequences that are cut, and the log sums."""
    import torch
    kw = _ways(kvr)[way]
    p = Problem(kvr, 95, "bf16", "bf16", [2000] * 32, [64] * 32, 8, 8, 64, 64)
    want = p.call()
    need = _workspace_bytes(kvr, p, 32)
    assert need > 1 << 24
    pending = Pending([2 * p.q.numel(), need] + [4 * p.q.shape[0] * p.q.shape[1]] * lse)
    got = p.call(want_lse=lse, stream=pending.side, **kw)
    pending.check(*(((got[0], want[0]),) if lse else ((got, want[0]),)))
    if lse:
        assert torch.equal(got[1], want[1])
