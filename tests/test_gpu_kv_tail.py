"""Half-precision caches keep the tail of the softmax: many tokens of little weight beside
one that dominates."""
import math

import numpy as np
import pytest

from tests.test_gpu_kv_attention import Problem
from tests.test_gpu_kv_cache import _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


# new tokens and queries a head: few rows, two row tiles a wave, rows that share tokens, blocks of 128
@pytest.mark.parametrize("nq,group", [(1, 4), (3, 8), (5, 8), (9, 12)])
@pytest.mark.parametrize("weight", [2.0 ** -15, 2.0 ** -20, 2.0 ** -26, 2.0 ** -30])
@pytest.mark.parametrize("sink", [0, 70001])
def test_one_token_dominates(kvr, nq, group, weight, sink):
    """Scores of all tokens are 0 but one's: its weight is 1, theirs ``weight`` (as near as half
    precision forms the score).  The dominant value is 1 in half of the head and 0 in the
    other; theirs is 3 and 1, so the other half is the tail's weight alone.  64 sequences of the
    same tokens and 8 KV heads, so that none is cut."""
    import torch
    n, dim, seqs = 131072, 64, 64
    p = Problem(kvr, 91, "fp16", "fp16", [n], [nq], 8, group, dim, 64)
    p.cu_q = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * nq
    p.kv_len, p.table, p.q = p.kv_len.repeat(seqs), p.table.repeat(seqs, 1), p.q.repeat(seqs, 1, 1)
    score = -math.log(weight)
    a = np.float16(math.sqrt(8 * score))             # scale is 1 / 8
    p.k.zero_()
    p.k[sink, :, 3] = float(a)
    p.v[:, :, :32], p.v[:, :, 32:] = 3.0, 1.0
    p.v[sink, :, :32], p.v[sink, :, 32:] = 1.0, 0.0
    p.q.zero_()
    p.q[:, :, 3] = float(a)
    kvr.kvr_cache_write(p.cache, p.k, p.v, p.slots)
    out, lse = p.call()
    assert all(torch.equal(x, x[:nq].repeat(seqs, *[1] * (x.dim() - 1))) for x in (out, lse))
    out, lse = _np(out[:nq]), _np(lse[:nq])
    w = math.exp(-float(a) ** 2 / 8)
    # rounded weights: to 2^-11 of themselves, or by 2^-25 of the least reference weight, 2^7;
    # scores and sums in 32 bits as in the attention tests, then the output's rounding
    for i in range(nq):
        others = n - nq + i                          # seen tokens without the dominant one
        total = 1 + others * w
        ds = (dim + 16) * 2.0 ** -24 * score
        rel = 2 * (2.0 ** -11 + 2 * ds + (n + 64) * 2.0 ** -24 + 2.0 ** -21)
        for want, x in (((1 + 3 * others * w) / total, out[i, :, :32]), (others * w / total, out[i, :, 32:])):
            tail = others * w / total * rel + others * 2.0 ** -32
            tol = tail * 3 + (want * 2.0 ** -11 + 2.0 ** -25) + want * 2.0 ** -11
            assert (np.abs(x - want) <= tol).all(), (i, want, float(np.abs(x - want).max()), tol)
        assert (np.abs(lse[i] - (float(a) ** 2 / 8 + math.log(total))) <=
                ds + (n + 64) * 2.0 ** -24 + 2.0 ** -20 * (1 + score)).all()
