"""kvr_latent_attention against the plain 64-bit definition: formats, sizes, lengths, pages,
masks, hidden values that are not numbers, workspaces, repeated calls."""
import math

import numpy as np
import pytest

from tests.latent_problem import LatentProblem, check_rows
from tests.test_gpu_kv_cache import _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


FORMATS = ["bf16", "fp16", "fp8"]
LAYOUTS = [  # heads, rank, rot, page
    (16, 512, 64, 16), (1, 256, 32, 16), (20, 512, 32, 32), (40, 256, 64, 64), (128, 512, 64, 16), (7, 256, 64, 256),
    (33, 512, 64, 64), (64, 256, 32, 32),
]


@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda x: "x".join(map(str, x)))
@pytest.mark.parametrize("fmt", FORMATS)
def test_decode(kvr, fmt, layout):
    """One new token of sequences from one cached token on, lengths around the tiles."""
    heads, rank, rot, page = layout
    p = LatentProblem(kvr, 31, fmt, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 128, 129, 517], [1] * 15, heads, rank, rot,
                      page, order="tpr" if heads == 20 else "ptr", slack=32)
    p.check(*p.call())


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda x: "x".join(map(str, x)))
@pytest.mark.parametrize("fmt", FORMATS)
def test_drafts(kvr, fmt, layout, tree):
    """Runs and trees of up to 70 new tokens, sequences without any, and ones that are new
    from their first token on."""
    heads, rank, rot, page = layout
    p = LatentProblem(kvr, 32, fmt, [70, 5, 0, 40, 33, 300, 64, 1], [70, 5, 0, 0, 2, 37, 64, 1], heads, rank, rot, page,
                      tree=tree)
    p.check(*p.call())


@pytest.mark.parametrize("nq", [1, 3, 9])
@pytest.mark.parametrize("fmt,rank", [("bf16", 512), ("fp16", 256), ("fp8", 512), ("bf16", 256)])
def test_long_sequences_are_cut_and_joined(kvr, fmt, rank, nq):
    import torch
    p = LatentProblem(kvr, 33, fmt, [20011, 700, 9000], [nq, nq, 0], 16, rank, 64, 64, tree=nq > 1)
    first = p.call()
    p.check(*first, rows=12)
    for _ in range(2):
        again = p.call()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_many_sequences(kvr):
    """More sequences than a wave has lanes, of very different lengths."""
    rng = np.random.default_rng(4)
    kv = [int(x) for x in np.exp(rng.uniform(0, math.log(1500), 150))]
    for heads in (8, 24):
        p = LatentProblem(kvr, 34, "fp8", kv, [min(t, int(rng.integers(0, 4))) for t in kv], heads, 256, 32, 16)
        p.check(*p.call(), rows=6)


@pytest.mark.parametrize("heads", [3, 9, 30])
@pytest.mark.parametrize("fmt", FORMATS)
def test_empty_rows_and_any_mask(kvr, fmt, heads):
    """Masks that leave rows empty (nothing cached before the drafts), hide a token from
    itself, and show later ones."""
    import torch
    p = LatentProblem(kvr, 35, fmt, [40, 12, 130], [40, 3, 30], heads, 256, 64, 16, tree=True)
    m = torch.from_numpy(np.random.default_rng(1).integers(-2 ** 62, 2 ** 62, p.mask.shape)).cuda()
    m[::3] = 0
    p.mask = m
    out, lse = p.call()
    p.check(out, lse)
    assert float(out[0].abs().max()) == 0 and bool((lse[0] == -math.inf).all())


@pytest.mark.parametrize("words", [2, 3])
def test_masks_of_several_words(kvr, words):
    p = LatentProblem(kvr, 36, "bf16", [300, 129], [100, 129], 2, 512, 64, 16, tree=True, words=max(words, 3))
    p.check(*p.call())


@pytest.mark.parametrize("nq,heads", [(20, 1), (20, 2), (20, 4), (37, 16)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_hidden_tokens_may_hold_anything(kvr, fmt, nq, heads):
    """Infinities and NaN in drafted tokens that some rows do not see, in the rows past the
    end of the last page, and in pages that are not in use."""
    import torch
    p = LatentProblem(kvr, 37, fmt, [900, 37], [nq, 37], heads, 512, 64, 16, tree=True)
    base = int(p.first[1])
    last = 900 - nq
    for t, d, value in ((last + 5, 540, math.inf), (last + 2, 5, math.nan), (last + 10, 5, math.inf),
                        (last + 13, 300, -math.inf), (base + 9, 7, math.nan), (base + 20, 511, -math.inf),
                        (base + 30, 530, math.nan)):
        p.rows[t, d] = value
    p.write()
    out, lse = p.call()
    p.check(out, lse, rows=400)
    assert bool(torch.isnan(out).any()) and bool(torch.isfinite(out).any(-1).any())


def test_seen_infinities(kvr):
    """A token of the past with an infinity: every row sees it."""
    p = LatentProblem(kvr, 38, "bf16", [100], [1], 4, 256, 32, 16)
    p.rows[7, 3] = math.inf
    p.write()
    p.check(*p.call())


@pytest.mark.parametrize("scale", [0.0, -0.07, 3.0])
def test_scales(kvr, scale):
    p = LatentProblem(kvr, 39, "bf16", [90, 1], [3, 1], 5, 256, 64, 32)
    p.scale = scale
    p.check(*p.call())


def test_a_dominant_token_among_many(kvr):
    """Half-precision weights beside one that is far larger."""
    p = LatentProblem(kvr, 40, "fp16", [40000], [1], 2, 256, 64, 64)
    p.rows[12345] *= 4
    p.write()
    p.check(*p.call(), rows=4)


def test_lengths_that_do_not_fit(kvr):
    """Left out and reported; the others are answered."""
    import torch
    p = LatentProblem(kvr, 41, "bf16", [60, 50, 70, 40], [2, 2, 2, 2], 16, 256, 32, 16)
    keep = p.kv_len.clone()
    for at, bad in ((1, 1), (1, 71), (2, 10000), (3, -5)):
        p.kv_len.copy_(keep)
        p.kv_len[at] = bad
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.full((8, 16, 256), 7.0, device="cuda").bfloat16()
        _, lse = p.call(status=status, check=False, out=out)
        assert int(status.item()) == kvr.KVR_E_DOMAIN
        p.check(out, lse, skip=(at,))
        assert bool((out[2 * at:2 * at + 2] == 7).all())
    p.kv_len.copy_(keep)
    p.table[0, 1] = 1 << 20   # a page outside the pool
    with pytest.raises(kvr.KvrError) as e:
        p.call()
    assert e.value.code == kvr.KVR_E_DOMAIN


def test_first_queries_that_decrease(kvr):
    """Half of the sequences have all the queries, the others fewer than none."""
    import torch
    p = LatentProblem(kvr, 42, "bf16", [1024], [16], 16, 256, 64, 64)
    n = 255
    p.cu_q = torch.tensor([0, 16] * 128, dtype=torch.int32, device="cuda")
    p.kv_len = torch.full((n,), 1024, dtype=torch.int32, device="cuda")
    p.table = p.table.repeat(n, 1)
    room = torch.full((1 << 30,), 0xFF, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = p.call(workspace=room, status=status, check=False)
    assert int(status.item()) == kvr.KVR_E_DOMAIN
    p.check(out, lse)   # all that are answered have the same tokens


def test_strided_queries_and_outputs(kvr):
    import torch
    p = LatentProblem(kvr, 43, "bf16", [77, 30], [4, 2], 3, 256, 32, 16)
    want = p.call()
    wide = torch.zeros(3, 6, 320, dtype=torch.bfloat16, device="cuda")
    wide[:, :, 16:304] = p.q.transpose(0, 1)
    p.q = wide[:, :, 16:304].transpose(0, 1)
    out = torch.zeros(6, 5, 264, dtype=torch.bfloat16, device="cuda")[:, 1:4, :256]
    got = p.call(out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_pages_beyond_32_bits(kvr):
    """A pool whose byte offsets pass 2^32: the last page is used."""
    import torch
    pages = (1 << 32) // (576 * 2 * 64) + 40
    cache = kvr.LatentCache(torch.empty(pages, 64, 576, dtype=torch.bfloat16, device="cuda"), 64)
    x = torch.randn(64, 576, device="cuda").bfloat16()
    slots = torch.arange(64, device="cuda") + (pages - 1) * 64
    kvr.kvr_latent_write(cache, x[:, :512], x[:, 512:], slots)
    assert torch.equal(kvr.kvr_latent_read(cache, slots), x)
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.randn(1, 16, 576, device="cuda").bfloat16()
    out = kvr.kvr_latent_attention(cache, q, torch.tensor([0, 1], **i32), torch.tensor([64], **i32),
                                   torch.tensor([[pages - 1]], **i32), 1, 64, 0.04)
    p = torch.softmax(q[0].double() @ x.double().T * 0.04, -1)
    want = p @ x[:, :512].double()
    # weights and outputs rounded to 2^-8 of themselves
    assert float(((out[0].double() - want).abs() - 2.0 ** -8 * (want.abs() + 1.01 * p @ x[:, :512].double().abs())).max()) <= 0


@pytest.mark.parametrize("fmt,heads,rank,n", [("bf16", 4, 256, 299), ("fp8", 20, 512, 150), ("fp16", 64, 256, 70),
                                              ("bf16", 70, 512, 75), ("bf16", 3, 256, 1100)])
def test_many_sequences_and_long_ones(kvr, fmt, heads, rank, n):
    """More row blocks than half of the CUs: parts of several rounds, beside sequences that are not cut."""
    rng = np.random.default_rng(n)
    kv = [int(x) for x in np.exp(rng.uniform(0, np.log(60), n))]
    kv[n // 2], kv[-1] = 9000, 3001
    p = LatentProblem(kvr, 50 + n, fmt, kv, [1] * n, heads, rank, 32, 16)
    p.check(*p.call(), rows=3)


@pytest.mark.parametrize("n,tokens", [(130, 700), (200, 300), (260, 530)])
def test_equal_sequences_of_several_rounds(kvr, n, tokens):
    p = LatentProblem(kvr, n, "bf16", [tokens] * n, [1 + b % 2 for b in range(n)], 8, 256, 64, 64)
    p.check(*p.call(), rows=3)


@pytest.mark.parametrize("fmt,rank", [("bf16", 256), ("fp16", 256), ("fp8", 256), ("bf16", 512), ("fp8", 512)])
@pytest.mark.parametrize("heads,q", [(12, 4), (24, 3), (16, 5), (20, 4), (13, 10), (16, 9), (59, 3), (20, 13)])
def test_rows_divided_among_blocks(kvr, fmt, rank, heads, q):
    """Rows that fill no whole block, of sequences that have more and fewer of them, with trees, and a
    hidden latent that is not finite."""
    import torch
    p = LatentProblem(kvr, 7 * heads + q, fmt, [q + 30, 700, 1 + q // 2, 333], [q, q, 1 + q // 2, 1], heads, rank, 64, 16, tree=True)
    p.check(*p.call(), rows=60)
    if fmt == "fp8":
        return
    # the last token of the second sequence, which only its own query sees
    t = torch.arange(q, device="cuda")
    p.mask[int(p.cu[1]):int(p.cu[2]), 0] = (2 << t) - 1
    p.rows[int(p.first[2]) - 1, 3] = float("nan")
    p.write()
    out, lse = p.call()
    assert bool(torch.isnan(out[int(p.cu[2]) - 1]).any()) and not bool(torch.isnan(out[:int(p.cu[2]) - 1]).any())
    p.check(out, lse, rows=30)


@pytest.mark.parametrize("rank,heads,q", [(512, 64, 40), (256, 128, 37), (512, 128, 17)])
def test_more_row_blocks_than_an_xcd_has(kvr, rank, heads, q):
    p = LatentProblem(kvr, rank + q, "bf16", [900, 333, q], [q, 1, q], heads, rank, 64, 64)
    p.check(*p.call(), rows=60)


@pytest.mark.parametrize("heads,rank,q", [(4, 512, 1), (16, 256, 1), (20, 512, 1), (64, 512, 1), (64, 256, 1), (128, 512, 1),
                                          (128, 256, 1), (20, 256, 7), (6, 512, 9)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_seen_infinities_everywhere(kvr, fmt, heads, rank, q):
    """One infinity in each 32 tokens of the past, each in a column of its own, whole parts of odd
    numbers of steps and tiles that hold the first new token among them.  Their scores are -infinity,
    so that they have no weight, and give NaN in those columns and nowhere else; for head 0 they are
    infinity, and everything is NaN."""
    import torch
    p = LatentProblem(kvr, 60 + heads, fmt, [32 * (rank - 9), 100, 64 + q, 1000, 224], [q] * 5, heads, rank, 64, 16)
    sign = 1 - 2 * (torch.arange(rank, device="cuda") % 2)
    x = p.q[..., :rank]
    x.copy_(x.abs().clamp(min=0.05) * sign)
    x[:, 0] = -x[:, 0]
    for b, t in enumerate(p.kv):
        s = torch.arange(-(-t // 32), device="cuda")
        at = 32 * s + 7 * s % 32
        s, at = s[at < t - q], at[at < t - q]
        slot = p.slots[int(p.first[b]) + at]
        page, off = slot // 16, slot % 16
        if fmt == "fp8":   # two times 2^127, alone in its block
            for i in range(32):
                p.cache.rows[page, off, s // 32 * 32 + i] = 0
            p.cache.rows[page, off, s] = torch.where(sign[s] > 0, 0xC0, 0x40).to(torch.uint8)
            p.cache.scale[page, off, s // 32] = 254
        else:
            p.cache.rows[page, off, s] = (-sign[s] * math.inf).to(p.cache.rows.dtype)
    out, lse = (_np(x) for x in p.call())
    rows, queries = _np(kvr.kvr_latent_read(p.cache, p.slots, torch.float32)), _np(p.q)
    for b, (t, n) in enumerate(zip(p.kv, p.nq)):
        xx, seen = rows[p.first[b]:p.first[b + 1]], p.seen(b)
        odd = ~np.isfinite(xx)
        gone, columns = odd.any(1), odd.any(0)[:rank]
        assert gone.sum() == columns.sum() >= (t - q) // 32 and not odd[:, rank:].any()
        seen = seen & ~gone
        for i in range(n):
            at = int(p.cu[b]) + i
            assert np.isnan(out[at, 0]).all(), (b, i)
            assert np.array_equal(np.isnan(out[at, 1:]), np.broadcast_to(columns, (heads - 1, rank))), (b, i)
        for h in {1, heads // 2, heads - 1}:
            own = slice(p.cu[b], p.cu[b + 1])
            check_rows(out[own, h][:, ~columns], lse[own, h], queries[own, h], xx, xx[:, :rank][:, ~columns], seen, p.scale,
                       p.dim, p.dtype, "fp16" if fmt == "fp16" else "bf16", (b, h))
