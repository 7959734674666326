"""Attention with up to 32 rows of a KV head, where every wave has all of them: one and two row
tiles, four and eight waves, in one launch and cut into parts; each with runs, trees, masks
that leave rows empty, and hidden values that are not finite."""
import math

import numpy as np
import pytest

from tests.test_gpu_kv_attention import Problem
from tests.test_gpu_kv_bounds import _workspace_bytes

pytestmark = pytest.mark.gpu

FORMATS = [("bf16", "bf16"), ("fp16", "fp16"), ("fp8", "bf16"), ("fp8", "fp16"), ("fp4", "bf16"), ("fp4", "fp16")]
# new tokens and queries a head
TWO_TILES = [(17, 1), (8, 3), (31, 1), (4, 8), (1, 32)]
ONE_TILE = [(4, 4), (1, 16), (5, 3), (16, 1)]


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


def _problem(kvr, seed, fmt, dtype, shape, dim, cut, tree=True, page=16):
    """Sequences that begin with their new tokens, and ones with older tokens; the plan is the
    one that the test is about."""
    nq, group = shape
    kv = [nq, nq + 9, 3001, 700] if cut else [nq, nq + 9, 65, 300, 512]
    p = Problem(kvr, seed, fmt, dtype, kv, [nq] * len(kv), 2, group, dim, page, tree=tree)
    rows = nq * group
    assert rows <= 16 or (rows <= 32 and dim <= 128)
    assert (_workspace_bytes(kvr, p, len(kv)) > 0) == cut
    if not cut and rows <= 16:
        assert 2 * len(kv) <= 256      # eight waves a block
    return p


def _shapes(dim):
    return ONE_TILE + (TWO_TILES if dim <= 128 else [])


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_runs_and_trees(kvr, fmt, dtype, dim, cut):
    for at, shape in enumerate(_shapes(dim)):
        for tree in (False, True):
            p = _problem(kvr, 101 + at, fmt, dtype, shape, dim, cut, tree)
            p.check(*p.call(), rows=5)


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_any_mask(kvr, fmt, dtype, dim, cut):
    """Random bits, and none at all for every third row: with no older tokens it sees nothing."""
    import torch
    for at, shape in enumerate(_shapes(dim)):
        p = _problem(kvr, 121 + at, fmt, dtype, shape, dim, cut)
        m = torch.from_numpy(np.random.default_rng(at).integers(-2 ** 62, 2 ** 62, p.mask.shape)).cuda()
        m[::3] = 0
        p.mask = m
        out, lse = p.call()
        p.check(out, lse, rows=5)
        empty = torch.arange(0, shape[0], 3, device="cuda")      # of the first sequence, which is all new
        assert int(out[empty].count_nonzero()) == 0 and bool((lse[empty] == -math.inf).all())


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_hidden_tokens_may_hold_anything(kvr, fmt, dtype, dim, cut):
    """Infinities and NaN in new tokens that no row or only some rows see."""
    import torch
    for at, shape in enumerate(_shapes(dim)):
        nq = shape[0]
        if nq < 4:
            continue
        p = _problem(kvr, 141 + at, fmt, dtype, shape, dim, cut)
        for b in range(len(p.kv)):
            first = int(p.first[b + 1]) - nq
            for x, t, head, d, value in ((p.k, 1, 0, 3, math.nan), (p.k, 1, 1, 9, math.inf), (p.v, 1, 0, 7, math.nan),
                                         (p.v, 1, 1, dim - 1, -math.inf), (p.v, 2, 0, 0, math.inf), (p.v, 2, 1, 40, math.nan)):
                x[first + t, head, d] = value
        kvr.kvr_cache_write(p.cache, p.k, p.v, p.slots)
        words = [(2 << i) - 1 & ~2 & ~4 | (4 if i == nq - 1 else 0) for i in range(nq)]   # token 2: the last row only
        p.mask = torch.tensor(words * len(p.kv), dtype=torch.int64, device="cuda")[:, None]
        out, lse = p.call()
        p.check(out, lse, rows=5)
        last = torch.arange(out.shape[0], device="cuda") % nq == nq - 1
        assert bool(torch.isfinite(out[~last]).all()) and bool(torch.isfinite(lse[~last]).all())
        assert not bool(torch.isfinite(out[last]).flatten(1).all(1).any())
