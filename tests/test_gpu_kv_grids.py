"""Calls of more than 2^32 threads, within the documented sizes."""
import numpy as np
import pytest

from tests import kv_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


@pytest.fixture(autouse=True)
def free_memory():
    import torch
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_rotary_table(kvr):
    n, rot = (1 << 25) + 3, 256
    table = kvr.kvr_rotary_table(rot, n, 500000.0)
    at = np.array([0, 1, 12345, (1 << 24) + 1, (1 << 25) - 1, 1 << 25, (1 << 25) + 2])
    a = at[:, None] * ref.frequencies(rot, 500000.0)
    got = table[at.tolist()].double().cpu().numpy()
    # the frequency's own rounding (a few 2^-53) times the angle, then one 32-bit rounding
    tol = 2.0 ** -24 + 16 * 2.0 ** -53 * (1 + a)
    assert (np.abs(got[:, 0] - np.cos(a)) <= tol).all() and (np.abs(got[:, 1] - np.sin(a)) <= tol).all()


def test_rotary(kvr):
    """One row for all tokens (a stride of 0), a size that goes one pair at a time."""
    import torch
    n, dim = (1 << 24) + 3, 258
    x = torch.randn(1, 1, dim, device="cuda").bfloat16().expand(n, 1, dim)
    table = kvr.kvr_rotary_table(2, 64)
    pos = torch.arange(n, device="cuda").int() % 64
    got = kvr.kvr_rotary(x, pos, table)
    for a in (0, 5000, n - 130):
        assert torch.equal(got[a:a + 130], kvr.kvr_rotary(x[a:a + 130], pos[a:a + 130], table))


def test_write_and_read(kvr):
    """All tokens but a few are written nowhere, and read as zeros."""
    import torch
    n, dim = (1 << 27) + 5, 256
    cache = kvr.KvCache.allocate(kvr.KVR_KV_BF16, 2, 1, 16, dim)
    x = torch.randn(1, 1, dim, device="cuda").bfloat16()
    slots = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    at = [0, 77, n - 6, n - 5, n - 1]
    slots[at] = torch.tensor([3, 4, 20, 21, 31], device="cuda")
    kvr.kvr_cache_write(cache, x.expand(n, 1, dim), x.expand(n, 1, dim), slots)
    rows = cache.k.reshape(32, dim)
    assert torch.equal(rows[[3, 4, 20, 21, 31]], x[0].expand(5, dim))
    assert int(rows.count_nonzero()) == 5 * int(x.count_nonzero())
    assert torch.equal(cache.v, cache.k)
    out = torch.empty((n, 1, dim), dtype=torch.bfloat16, device="cuda")
    kvr.kvr_cache_read(cache, slots, out=(out, out))
    assert torch.equal(out[at, 0], x[0].expand(5, dim))
    others = [1, 76, 78, 1 << 26, n - 7, n - 4, n - 2]
    assert int(out[others].count_nonzero()) == 0
