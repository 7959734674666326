"""Quantised blocks whose values reach 2^128, and so are infinities in 32 bits: they read
back as such, and attention's rows that do not see them are not touched."""
import numpy as np
import pytest

from tests import kv_reference as ref
from tests.test_gpu_kv_attention import Problem
from tests.test_gpu_kv_cache import _cache, _dt, _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_largest_scales_read_back(kvr, fmt):
    """All codes under every scale byte from 245 on."""
    import torch
    cache = _cache(kvr, fmt, 1, 11, 16, 256, fill=0)
    n = 256 if fmt == "fp8" else 16
    codes = np.tile(np.arange(n, dtype=np.uint8), 11 * 16 * 256 // n).reshape(1, 11, 16, 256)
    scale = np.broadcast_to(np.arange(245, 256, dtype=np.uint8)[None, :, None, None], (1, 11, 16, 8)).copy()
    for data in (cache.k, cache.v):
        data.copy_(torch.from_numpy(ref.pack(codes, fmt)))
    for data in (cache.k_scale, cache.v_scale):
        data.copy_(torch.from_numpy(scale))
    slots = torch.arange(16, device="cuda")
    for dt in ("fp32", "bf16", "fp16"):
        k, v = kvr.kvr_cache_read(cache, slots, _dt(dt))
        want = torch.from_numpy(ref.dequantise(codes, scale, fmt)[0].transpose(1, 0, 2)).to(_dt(dt)).double().numpy()
        assert np.array_equal(_np(k), want, equal_nan=True) and torch.equal(k.view(torch.uint8), v.view(torch.uint8))
    assert np.isinf(want).any()


# new tokens, queries a head, head size, cached tokens: few rows in one launch (eight waves), few rows
# cut, 17 to 32 rows uncut and cut, more rows that share tokens
SHAPES = [(4, 4, 64, 90), (5, 3, 96, 300), (4, 4, 256, 40), (4, 3, 128, 5000), (8, 4, 128, 100), (6, 4, 96, 7000),
          (17, 1, 64, 40), (20, 4, 128, 90), (20, 1, 192, 300), (40, 8, 64, 9000)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("fmt,dtype", [("fp8", "bf16"), ("fp8", "fp16"), ("fp4", "bf16"), ("fp4", "fp16")])
def test_hidden_values_that_overflow(kvr, fmt, dtype, shape):
    """One drafted token, key and value, that no row sees; one value that only some rows see;
    and the rows past the end and the unused pages: scale bytes from 247 (e4m3) or 253
    (e2m1) on with codes that reach 2^128, zeros, and for e4m3 small codes beside them."""
    import torch
    nq, group, dim, kv = shape
    fill = 0xF8 if fmt == "fp8" else 0xFD     # -256 * 2^121; -6 and -3 * 2^126
    p = Problem(kvr, 81, fmt, dtype, [kv, nq], [nq, nq], 2, group, dim, 16, tree=True, fill=fill)
    unseen, some, after = 1, 2, nq - 1
    rng = np.random.default_rng(5)
    low = 247 if fmt == "fp8" else 253
    big, small = ([0x78, 0x7E, 0xF8, 0xFE], [0, 0x80]) if fmt == "fp8" else ([6, 7, 14, 15], [0, 8])
    if fmt == "fp8" and dtype == "bf16":
        small += [1, 2, 0x83]                 # below 2^119: finite beside the infinities
    for b in range(2):
        for token, names in ((unseen, "kv"), (some, "v")):
            slot = int(p.slots[int(p.first[b]) + kv * (b == 0) + nq * (b == 1) - nq + token])
            for name in names:
                codes = rng.choice(big + small, (2, dim)).astype(np.uint8)
                codes[:, ::32] = big[0]
                data, scale = getattr(p.cache, name), getattr(p.cache, name + "_scale")
                data[slot // 16, :, slot % 16] = torch.from_numpy(ref.pack(codes, fmt)).cuda()
                scale[slot // 16, :, slot % 16] = torch.from_numpy(
                    rng.integers(low, 255, (2, dim // 32)).astype(np.uint8)).cuda()
    words = []
    for i in range(nq):
        seen = (2 << i) - 1 & ~(1 << unseen) & ~(1 << some)
        words.append(seen | (1 << some if i == after else 0))
    p.mask = torch.tensor(words + words, dtype=torch.int64, device="cuda")[:, None]
    out, lse = p.call()
    p.check(out, lse)
    clean = [i for i in range(2 * nq) if i % nq != after]
    assert bool(torch.isfinite(out[clean]).all()) and bool(torch.isfinite(lse[clean]).all())
    assert bool(torch.isinf(out[after]).any())
