"""kvr_latent_write and kvr_latent_read against the plain definitions: formats, types, norms,
rotations, strides, slots that are skipped or outside the pool."""
import numpy as np
import pytest

from tests import kv_reference as ref
from tests.latent_problem import EPS, make_cache
from tests.test_gpu_kv_cache import _dt, _np, _randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


SIZES = [(512, 64), (256, 32), (512, 32), (256, 64)]


def _slots(rng, tokens, pages, page):
    import torch
    return torch.from_numpy(rng.permutation(pages * page)[:tokens].astype(np.int64)).cuda()


def _expect16(x, fmt):
    """Rounded to the format once, from 32 bits."""
    import torch
    return torch.from_numpy(np.asarray(x, np.float32)).to(_dt(fmt)).double().numpy()


@pytest.mark.parametrize("tokens", [1, 7, 67, 9001])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("fp16", "fp16"), ("fp8", "bf16"), ("bf16", "fp32"), ("fp8", "fp16")])
def test_rows_as_they_are(kvr, fmt, dtype, size, tokens):
    """No norm, no rotation: rounded once, which is exact here or a code of the block."""
    import torch
    rank, rot = size
    rng = np.random.default_rng(tokens)
    pages, page = tokens // 16 + 2, 16
    cache = make_cache(kvr, fmt, pages, page, rank, rot, fill=0xFF, order="tpr" if rot == 32 else "ptr", slack=16)
    x = _randn(1, (tokens, rank + rot), dtype)
    slots = _slots(rng, tokens, pages, page)
    slots[::5] = -1
    before = cache.rows.clone()
    kvr.kvr_latent_write(cache, x[:, :rank], x[:, rank:], slots)
    got = _np(kvr.kvr_latent_read(cache, slots, torch.float32))
    live = (slots >= 0).cpu().numpy()
    if fmt == "fp8":
        codes, scale = ref.quantise(_np(x[:400]), "fp8")
        want = ref.dequantise(codes, scale, "fp8")
    else:
        want = _expect16(_np(x[:400]), fmt)
    want[~live[:400]] = 0
    assert np.array_equal(got[:400], want)
    assert (got[~live] == 0).all()
    # nothing else has been written
    touched = torch.zeros(pages * page, dtype=torch.bool, device="cuda")
    touched[slots[slots >= 0]] = True
    same = (cache.rows.view(torch.uint8) == before.view(torch.uint8)).all(-1).reshape(-1)
    assert bool(same[~touched].all())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot_dim", [64, 20, 32])
@pytest.mark.parametrize("tokens", [5, 8200])
@pytest.mark.parametrize("fmt", ["bf16", "fp16", "fp8"])
def test_norm_and_rotation(kvr, fmt, tokens, rot_dim, interleaved):
    import torch
    rank, rot, eps = 512, 64, 1e-5
    dtype = "fp16" if fmt == "fp16" else "bf16"
    pages, page = tokens // 32 + 2, 32
    rng = np.random.default_rng(3)
    cache = make_cache(kvr, fmt, pages, page, rank, rot)
    x = _randn(4, (tokens, rank + rot), dtype)
    w = _randn(5, (rank,), dtype)
    slots = _slots(rng, tokens, pages, page)
    pos = torch.from_numpy(rng.integers(0, 5000, tokens).astype(np.int32)).cuda()
    table = kvr.kvr_rotary_table(rot_dim, 5000)
    kvr.kvr_latent_write(cache, x[:, :rank], x[:, rank:], slots, pos, table, norm_weight=w, eps=eps,
                         interleaved=interleaved)
    got = _np(kvr.kvr_latent_read(cache, slots, torch.float32))[:300]
    c = _np(x[:300, :rank])
    latent = c * _np(w) / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    # the norm in 32 bits: a sum of `rank` squares, a root, a quotient, two products
    slip = (rank + 8) * 2.0 ** -24
    t = table[pos[:300].long()].cpu().numpy()
    key = _np(x[:300, rank:])[:, None]
    key[..., :rot_dim] = ref.rotate(key[..., :rot_dim], t[:, 0], t[:, 1], interleaved, dtype=np.float32)
    if fmt == "fp8":
        k = _np(cache.scale.reshape(-1, (rank + rot) // 32)[slots[:300]].float()) - 127
        half = np.repeat(np.ldexp(1.0, k.astype(int) - 10), 32, 1)   # half a step of the smallest codes
        tol = np.maximum(np.abs(latent) * (2.0 ** -4 + 2 * slip), half[:, :rank] * (1 + 2 * slip))
        codes, scale = ref.quantise(key[:, 0], "fp8")
        want = ref.dequantise(codes, scale, "fp8")
    else:
        tol = np.abs(latent) * (EPS[fmt] + 2 * slip) + (2.0 ** -25 if fmt == "fp16" else 0)
        want = _expect16(key[:, 0], fmt)
    assert (np.abs(got[:, :rank] - latent) <= tol).all()
    assert np.array_equal(got[:, rank:], want)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_values_that_are_not_numbers(kvr, fmt):
    """A NaN or an infinity stays in its element (16 bits) or its block (codes); with a norm in its
    row's latent, and never in other rows."""
    import torch
    rank, rot = 256, 32
    x = _randn(7, (40, rank + rot), "bf16")
    x[3, 5], x[9, rank + 1], x[17, 40] = float("nan"), float("inf"), -float("inf")
    slots = torch.arange(40, device="cuda")
    cache = make_cache(kvr, fmt, 3, 16, rank, rot)
    kvr.kvr_latent_write(cache, x[:, :rank], x[:, rank:], slots)
    got = _np(kvr.kvr_latent_read(cache, slots, torch.float32))
    bad = ~np.isfinite(got)
    want = np.zeros_like(bad)
    for t, d in ((3, 5), (9, rank + 1), (17, 40)):
        want[t, slice(d, d + 1) if fmt == "bf16" else slice(d // 32 * 32, d // 32 * 32 + 32)] = True
    assert np.array_equal(bad, want)
    kvr.kvr_latent_write(cache, x[:, :rank], x[:, rank:], slots, norm_weight=torch.ones(rank, device="cuda").bfloat16())
    bad = ~np.isfinite(_np(kvr.kvr_latent_read(cache, slots, torch.float32)))
    assert bad[3, :rank].any() and bad[17, :rank].any()
    assert not bad[[t for t in range(40) if t not in (3, 9, 17)]].any() and not bad[9, :rank].any()


def test_zero_rows_and_a_norm(kvr):
    """eps keeps a row of zeros from a division by zero; without it the row is NaN."""
    import torch
    x = torch.zeros(2, 576, device="cuda").bfloat16()
    cache = make_cache(kvr, "bf16", 1, 16, 512, 64)
    slots = torch.arange(2, device="cuda")
    w = torch.ones(512, device="cuda").bfloat16()
    kvr.kvr_latent_write(cache, x[:, :512], x[:, 512:], slots, norm_weight=w)
    assert float(kvr.kvr_latent_read(cache, slots).abs().max()) == 0
    kvr.kvr_latent_write(cache, x[:, :512], x[:, 512:], slots, norm_weight=w, eps=0.0)
    assert bool(torch.isnan(kvr.kvr_latent_read(cache, slots)[:, :512]).all())


@pytest.mark.parametrize("fmt", ["fp16", "fp8"])
@pytest.mark.parametrize("out", ["bf16", "fp16", "fp32"])
def test_read_types_and_slots(kvr, fmt, out):
    """Rows any number of times, zeros below 0; outside the pool zeros and an error."""
    import torch
    rank, rot, n = 512, 32, 3000
    cache = make_cache(kvr, fmt, 4, 16, rank, rot, order="tpr")
    x = _randn(8, (64, rank + rot), "fp16")
    kvr.kvr_latent_write(cache, x[:, :rank], x[:, rank:], torch.arange(64, device="cuda"))
    slots = torch.randint(-3, 64, (n,), device="cuda")
    whole = _np(kvr.kvr_latent_read(cache, torch.arange(64, device="cuda"), torch.float32))
    want = torch.from_numpy(np.where((slots >= 0).cpu().numpy()[:, None], whole[slots.clamp(min=0).cpu().numpy()], 0))
    room = torch.full((n, rank + rot + 8), 7.0, dtype=_dt(out), device="cuda")
    got = kvr.kvr_latent_read(cache, slots, out=room[:, :rank + rot])
    assert torch.equal(got.cpu().double(), want.to(_dt(out)).double()) and bool((room[:, rank + rot:] == 7).all())
    slots[5], slots[6] = 64, 1 << 40
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = kvr.kvr_latent_read(cache, slots, _dt(out), status=status, check=False)
    assert int(status.item()) == kvr.KVR_E_DOMAIN and float(got[5:7].abs().max()) == 0


def test_writes_outside_are_reported(kvr):
    import torch
    cache = make_cache(kvr, "bf16", 4, 16, 256, 64, fill=0)
    x = _randn(9, (3, 320), "bf16")
    table = kvr.kvr_rotary_table(64, 10)
    pos = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    ok = torch.tensor([3, 4, 5], device="cuda")
    for slots, p in ((torch.tensor([3, 64, 5], device="cuda"), pos), (ok, torch.tensor([1, 10, 3], dtype=torch.int32, device="cuda")),
                     (ok, torch.tensor([1, -1, 3], dtype=torch.int32, device="cuda"))):
        cache.rows.zero_()
        with pytest.raises(kvr.KvrError) as e:
            kvr.kvr_latent_write(cache, x[:, :256], x[:, 256:], slots, p, table)
        assert e.value.code == kvr.KVR_E_DOMAIN
        rows = kvr.kvr_latent_read(cache, ok)
        assert float(rows[1].abs().max()) == 0 and bool((rows[::2].abs().amax(1) > 0).all())
