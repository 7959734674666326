"""kvr_latent_prompt against the plain 64-bit definition: types, sizes, ragged lengths, chunks
behind a past, layouts, hidden values that are not numbers, keys cut into parts."""
import math

import pytest

from tests.latent_problem import PromptProblem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


SIZES = [(128, 64), (64, 32), (128, 32), (64, 64)]
EDGES = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 128, 129, 255, 257]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_prompts(kvr, dtype, size, causal):
    """Lengths around the tiles, and sequences without tokens."""
    p = PromptProblem(51, dtype, EDGES + [0, 300], EDGES + [0, 300], 2, 1, *size, causal=causal)
    p.check(*p.call(kvr))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_chunks_behind_a_past(kvr, dtype, size, causal):
    """Fewer queries than keys, grouped heads, heads first in memory."""
    p = PromptProblem(52, dtype, [1, 70, 5, 130, 0, 64], [200, 70, 64, 391, 50, 1000], 3, 2, *size, causal=causal, packed=False)
    p.check(*p.call(kvr))


@pytest.mark.parametrize("causal", [True, False])
def test_more_queries_than_keys(kvr, causal):
    """The first queries of a causal sequence then see nothing: zeros and -infinity."""
    import torch
    p = PromptProblem(53, "bf16", [100, 200, 5], [60, 0, 5], 2, 1, 64, 32, causal=causal)
    out, lse = p.call(kvr)
    p.check(out, lse)
    empty = torch.cat([torch.arange(40 if causal else 0), torch.arange(100, 300)])
    assert float(out[empty].abs().max()) == 0 and bool((lse[empty] == -math.inf).all())


@pytest.mark.parametrize("nq", [1, 3, 100])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_keys_cut_into_parts(kvr, dtype, nq):
    import torch
    p = PromptProblem(54, dtype, [nq, 2], [9001, 700], 2, 2, 128, 64)
    first = p.call(kvr)
    p.check(*first, rows=16)
    for _ in range(2):
        again = p.call(kvr)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_a_long_prompt(kvr):
    p = PromptProblem(55, "bf16", [3001, 1500], [3001, 2500], 8, 1, 128, 64)
    p.check(*p.call(kvr), rows=40)


def test_many_sequences(kvr):
    """More sequences than a wave has lanes."""
    n = [1 + (37 * i) % 90 for i in range(150)]
    p = PromptProblem(56, "fp16", n, [x + 11 * (i % 5) for i, x in enumerate(n)], 1, 3, 64, 64)
    p.check(*p.call(kvr), rows=6)


@pytest.mark.parametrize("nk", [150, 2100])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_hidden_keys_may_hold_anything(kvr, dtype, nk):
    """Infinities and NaN in later keys and values, and in the next sequence's."""
    import torch
    p = PromptProblem(57, dtype, [150, 20], [nk, 20], 2, 1, 128, 64)
    at = nk - 150
    for x, t, d, value in ((p.k, at + 70, 3, math.nan), (p.v, at + 90, 3, math.inf), (p.v, at + 100, 5, math.nan),
                           (p.v, at + 120, 100, -math.inf), (p.v, nk, 7, math.nan), (p.k, nk, 9, math.inf)):
        x[t, 0, d] = value
    p.k_rot[nk - 1, 2] = math.nan
    out, lse = p.call(kvr)
    p.check(out, lse, rows=600)
    assert bool(torch.isnan(out).any()) and bool(torch.isfinite(out[:70]).all())


@pytest.mark.parametrize("scale", [0.0, -0.1, 2.0])
def test_scales(kvr, scale):
    p = PromptProblem(58, "bf16", [90], [90], 2, 1, 64, 32)
    p.scale = scale
    p.check(*p.call(kvr))


def test_large_scores_move_the_reference(kvr):
    """Scores that grow along the keys, so that the running maximum moves all the time."""
    import torch
    for dtype in ("bf16", "fp16"):
        p = PromptProblem(59, dtype, [200], [900], 1, 1, 64, 32)
        ramp = torch.linspace(0, 12, 900, device="cuda")[:, None, None]
        p.q[:] = p.q.abs()
        p.k.copy_((p.k.abs().float() * ramp).to(p.k.dtype))
        p.check(*p.call(kvr), rows=60)


def test_lengths_that_do_not_fit(kvr):
    import torch
    p = PromptProblem(60, "bf16", [30, 40, 20], [50, 40, 90], 2, 1, 64, 32)
    want, _ = p.call(kvr)
    for change in (dict(max_q=39), dict(max_k=89)):
        keep = p.max_q, p.max_k
        for k, v in change.items():
            setattr(p, k, v)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.full_like(want, 7.0)
        p.call(kvr, status=status, check=False, out=out)
        p.max_q, p.max_k = keep
        assert int(status.item()) == kvr.KVR_E_DOMAIN
        gone = slice(30, 70) if "max_q" in change else slice(70, 90)
        assert bool((out[gone] == 7).all())
        out[gone] = want[gone]
        assert torch.equal(out, want)
    for bad in ([0, 30, 70, 95], [-1, 30, 70, 90], [0, 30, 20, 90]):
        cu = torch.tensor(bad, dtype=torch.int32, device="cuda")
        with pytest.raises(kvr.KvrError) as e:
            kvr.kvr_latent_prompt(p.q, p.k, p.k_rot, p.v, cu, p.cu_k, 90, 90)
        assert e.value.code == kvr.KVR_E_DOMAIN
        with pytest.raises(kvr.KvrError) as e:
            kvr.kvr_latent_prompt(p.q, p.k, p.k_rot, p.v, p.cu_q, 2 * cu, 40, 180)
        assert e.value.code == kvr.KVR_E_DOMAIN


def test_strides_and_outputs(kvr):
    import torch
    p = PromptProblem(61, "bf16", [70, 3], [70, 80], 2, 1, 64, 32)
    want = p.call(kvr)
    room = torch.full((73, 4, 72), 7.0, device="cuda").bfloat16()
    p.q = torch.cat([p.q, p.q], -1)[:, :, 96:]
    got = p.call(kvr, out=room[:, 1:3, :64])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    room[:, 1:3, :64] = 7
    assert bool((room == 7).all())
    plain = p.call(kvr, want_lse=False, scale=None)
    assert torch.equal(plain, want[0])
