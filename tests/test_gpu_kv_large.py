"""Calls beyond the sizes at which the kernels change their ways: outputs written past the
caches, many parts of one sequence, blocks of many rows; and masks of one word or two."""
import numpy as np
import pytest

from tests.test_gpu_kv_attention import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


def _random(seed, shape, dtype):
    import torch
    gen = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,dim,rot", [(9, 256, 256), (36, 64, 32), (24, 96, 48), (13, 192, 96)])
@pytest.mark.parametrize("dt", ["bfloat16", "float16", "float32"])
def test_large_rotary_is_many_small_ones(kvr, dt, heads, dim, rot, interleaved):
    """Tokens do not depend on one another: one call gives the bits of many."""
    import torch
    n = 20_000_003 // (heads * dim)
    x = _random(1, (n, heads, dim), getattr(torch, dt))
    table = kvr.kvr_rotary_table(rot, 5000)
    pos = (torch.arange(n, device="cuda") * 7 % 5000).int()
    y = kvr.kvr_rotary(x, pos, table, interleaved=interleaved)
    for a in range(0, n, 1999):
        part = kvr.kvr_rotary(x[a:a + 1999], pos[a:a + 1999], table, interleaved=interleaved)
        assert torch.equal(part, y[a:a + 1999]), a
    # the adjoint takes it back but for two roundings
    back = kvr.kvr_rotary(y, pos, table, interleaved=interleaved, adjoint=True)
    eps = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -22}[dt]
    pairs = x.float().abs().amax() * 2
    assert (back.float() - x.float()).abs().amax() <= 2 * eps * pairs
    assert kvr.kvr_rotary(x, pos, table, interleaved=interleaved, out=x) is x and torch.equal(x, y)


@pytest.mark.parametrize("heads,dim", [(9, 128), (5, 96), (3, 256)])
@pytest.mark.parametrize("out", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("fmt", ["BF16", "FP16", "FP8", "FP4"])
def test_large_read_is_many_small_ones(kvr, fmt, out, heads, dim):
    import torch
    n, page = 9_500_017 // (heads * dim), 64
    pages = -(-n // page) + 3
    cache = kvr.KvCache.allocate(getattr(kvr, "KVR_KV_" + fmt), pages, heads, page, dim)
    slots = torch.randperm(pages * page, device="cuda")[:n]
    src = torch.float16 if fmt == "FP16" else torch.bfloat16
    k, v = _random(3, (n, heads, dim), src), _random(4, (n, heads, dim), src)
    kvr.kvr_cache_write(cache, k, v, slots)
    slots[::50] = -1
    got = kvr.kvr_cache_read(cache, slots, getattr(torch, out))
    for a in range(0, n, 1501):
        part = kvr.kvr_cache_read(cache, slots[a:a + 1501], getattr(torch, out))
        for x, y in zip(part, got):
            assert torch.equal(x, y[a:a + 1501]), a
    assert int(got[0][::50].count_nonzero()) == 0
    if fmt in ("BF16", "FP16"):   # kept as they were
        assert torch.equal(got[1][1], v[1].to(getattr(torch, out)))


@pytest.mark.parametrize("fmt,dtype,dim", [("bf16", "bf16", 64), ("fp8", "fp16", 128), ("fp4", "bf16", 192),
                                           ("fp16", "fp16", 256)])
def test_one_long_sequence_of_one_head(kvr, fmt, dtype, dim):
    """Hundreds of parts of a few rows."""
    import torch
    p = Problem(kvr, 61, fmt, dtype, [50021], [2], 1, 3, dim, 256, tree=True)
    first = p.call()
    p.check(*first, rows=2)
    assert all(torch.equal(x, y) for x, y in zip(first, p.call()))


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("fp8", "bf16"), ("fp4", "fp16")])
@pytest.mark.parametrize("group,dim", [(8, 128), (2, 64), (1, 256), (3, 96)])
def test_short_sequences_of_many_rows(kvr, fmt, dtype, group, dim):
    """Parts are whole numbers of steps, about as many as fill the GPU, or none."""
    kv = [63, 64, 65, 95, 96, 97, 127, 160, 255, 256, 257, 511, 512, 513, 530, 800, 1025, 33, 40]
    p = Problem(kvr, 62, fmt, dtype, kv, [min(63, 9 + 5 * b) for b in range(len(kv) - 2)] + [33, 40], 2, group,
                dim, 16, tree=True)
    p.check(*p.call(), rows=6)


@pytest.mark.parametrize("group", [1, 5, 20])
@pytest.mark.parametrize("tree", [False, True])
def test_words_of_the_mask(kvr, group, tree):
    """The same masks in one word and in two, and the run of tokens as a mask, give the same
    bits; new tokens begin at every place of a step."""
    import torch
    nq = [1 + 7 * b % 64 for b in range(33)]
    kv = [n + b for b, n in enumerate(nq)]
    p = Problem(kvr, 63, "bf16", "bf16", kv, nq, 2, group, 64, 16, tree=True)
    if not tree:
        run = [(2 << i) - 1 for n in nq for i in range(n)]
        p.mask = torch.from_numpy(np.array([x - 2 ** 64 if x >> 63 else x for x in run], np.int64)[:, None]).cuda()
    assert p.mask.shape[1] == 1

    def call(mask):
        return kvr.kvr_tree_attention(p.cache, p.q, p.cu_q, p.kv_len, p.table, p.max_q, p.max_kv,
                                      tree_mask=mask, want_lse=True)

    one, two = call(p.mask), call(torch.cat([p.mask, torch.full_like(p.mask, -1)], 1))
    assert all(torch.equal(x, y) for x, y in zip(one, two))
    if not tree:
        assert all(torch.equal(x, y) for x, y in zip(one, call(None)))
    else:
        p.check(*one)


def test_rows_that_see_nothing(kvr):
    """Empty masks over sequences without older tokens: zeros and a log sum of -infinity."""
    import torch
    for group in (1, 8):   # few rows, and many
        p = Problem(kvr, 64, "fp8", "bf16", [40, 70], [40, 10], 2, group, 128, 16, tree=True)
        p.mask[:20] = 0
        out, lse = kvr.kvr_tree_attention(p.cache, p.q, p.cu_q, p.kv_len, p.table, p.max_q, p.max_kv,
                                          tree_mask=p.mask, want_lse=True)
        assert int(out[:20].count_nonzero()) == 0 and bool((lse[:20] == -float("inf")).all())
        assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse[20:]).all())
        assert int(out[20:].count_nonzero()) > 0


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("fp4", "fp16")])
@pytest.mark.parametrize("n,longest", [(20, 1023), (20, 1040), (70, 512), (70, 1024), (150, 520), (130, 2048), (130, 2060)])
def test_many_short_sequences(kvr, fmt, dtype, n, longest):
    """One new token: sequences that one block takes whole, and ones that are cut."""
    rng = np.random.default_rng(n)
    kv = [int(x) for x in np.exp(rng.uniform(0, np.log(longest), n))]
    kv[n // 2] = longest
    p = Problem(kvr, 65, fmt, dtype, kv, [1] * n, 8, 2, 64, 16)
    p.check(*p.call())


@pytest.mark.parametrize("group", [2, 8])
def test_many_trees_of_ragged_sizes(kvr, group):
    """More row blocks than one launch has room for in order of sequences."""
    n = 300
    nq = [64 if b % 25 == 0 else b % 4 for b in range(n)]
    kv = [q + (b * 13 % 60 if q else 0) for b, q in enumerate(nq)]
    p = Problem(kvr, 66, "bf16", "bf16", kv, nq, 1, group, 64, 16, tree=True)
    p.check(*p.call(), rows=4)
