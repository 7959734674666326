"""C-ABI checks of the KV cache's entry points that need no GPU: bad arguments are
refused with the documented codes before the device is touched, workspaces are
sized, empty calls succeed.  And the plain definitions of kv_reference, checked
against each other."""
import ctypes
import math
import os

import numpy as np
import pytest

import paper_2608_30830_amd as kvr
from tests import kv_reference as ref

FAKE = ctypes.c_void_p(0x1000)   # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kvr.LIB_PATH):
        from paper_2608_30830_amd import build
        build.build()
    return kvr.load_library()


def _cache(fmt=None, **kw):
    c = kvr.kvr_kv_cache(k_data=0x1000, v_data=0x2000, k_scale=0x3000, v_scale=0x4000,
                         page_stride=8 * 16 * 128, head_stride=16 * 128, token_stride=128,
                         scale_page_stride=512, scale_head_stride=64, scale_token_stride=4,
                         n_pages=10, page_size=16, n_kv_heads=8, head_dim=128,
                         format=kvr.KVR_KV_FP8 if fmt is None else fmt)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _write(lib, c, k=FAKE, v=FAKE, dt=0, n=4, st=(1024, 128, 1024, 128), slots=FAKE, pos=None, table=None,
           n_pos=0, rot=0, flags=0):
    return lib.kvr_cache_write(None if c is None else ctypes.byref(c), k, v, dt, n, *st, slots, pos, table,
                               n_pos, rot, flags, None, None)


BAD_CACHES = [
    (dict(k_data=None), kvr.KVR_E_NULL), (dict(v_scale=None), kvr.KVR_E_NULL),
    (dict(format=4), kvr.KVR_E_LAYOUT), (dict(format=-1), kvr.KVR_E_LAYOUT),
    (dict(n_pages=0), kvr.KVR_E_SIZE), (dict(n_pages=1 << 31), kvr.KVR_E_SIZE),
    (dict(n_kv_heads=0), kvr.KVR_E_SIZE), (dict(n_kv_heads=1025), kvr.KVR_E_SIZE),
    (dict(page_size=8), kvr.KVR_E_LAYOUT), (dict(page_size=48), kvr.KVR_E_LAYOUT),
    (dict(page_size=1 << 16), kvr.KVR_E_LAYOUT), (dict(head_dim=80), kvr.KVR_E_LAYOUT),
    (dict(head_dim=32), kvr.KVR_E_LAYOUT), (dict(head_dim=512), kvr.KVR_E_LAYOUT),
    (dict(v_data=0x2008), kvr.KVR_E_LAYOUT), (dict(token_stride=120), kvr.KVR_E_LAYOUT),
    (dict(page_stride=-16), kvr.KVR_E_LAYOUT), (dict(head_stride=8), kvr.KVR_E_LAYOUT),
    (dict(token_stride=1 << 27), kvr.KVR_E_LAYOUT), (dict(scale_token_stride=-1), kvr.KVR_E_LAYOUT),
]


@pytest.mark.parametrize("kw,code", BAD_CACHES, ids=lambda x: str(x))
def test_bad_caches(lib, kw, code):
    c = _cache(**kw)
    assert _write(lib, c) == code
    assert lib.kvr_cache_read(ctypes.byref(c), FAKE, 4, FAKE, FAKE, 0, 1024, 128, 1024, 128, None, None) == code
    assert _attend(lib, c) == code


def test_strides_of_one_element_do_not_matter(lib):
    c = _cache(n_pages=1, n_kv_heads=1, page_stride=-7, head_stride=3, scale_page_stride=-1, scale_head_stride=-1)
    assert _write(lib, c, n=0) == kvr.KVR_OK
    assert _write(lib, c, slots=None, n=1, st=(3, 5, -1, 7)) == kvr.KVR_E_NULL
    assert _write(lib, _cache(), k=ctypes.c_void_p(0x1002)) == kvr.KVR_E_LAYOUT


def test_write_and_read_refusals(lib):
    c = _cache()
    assert _write(lib, None) == kvr.KVR_E_NULL
    assert _write(lib, c, n=-1) == kvr.KVR_E_SIZE
    assert _write(lib, c, n=1 << 29) == kvr.KVR_E_SIZE
    assert _write(lib, c, dt=3) == kvr.KVR_E_LAYOUT
    assert _write(lib, c, n=0) == kvr.KVR_OK
    assert _write(lib, c, n=0, k=None, v=None, slots=None) == kvr.KVR_OK
    for kw in (dict(k=None), dict(v=None), dict(slots=None)):
        assert _write(lib, c, **kw) == kvr.KVR_E_NULL
    for st in ((1023, 128, 1024, 128), (1024, 120 + 4, 1024, 128), (1024, 128, -8, 128)):
        assert _write(lib, c, st=st) == kvr.KVR_E_LAYOUT
    assert _write(lib, c, table=FAKE, n_pos=9, rot=128) == kvr.KVR_E_NULL          # no positions
    for rot in (0, 3, 130, -2):
        assert _write(lib, c, pos=FAKE, table=FAKE, n_pos=9, rot=rot) == kvr.KVR_E_SIZE
    assert _write(lib, c, pos=FAKE, table=FAKE, n_pos=0, rot=128) == kvr.KVR_E_SIZE
    assert _write(lib, c, pos=FAKE, table=ctypes.c_void_p(0x1002), n_pos=9, rot=128) == kvr.KVR_E_LAYOUT
    assert _write(lib, c, pos=FAKE, table=FAKE, n_pos=9, rot=128, flags=4) == kvr.KVR_E_METHOD
    read = lambda k=FAKE, n=4, dt=0, s=FAKE: lib.kvr_cache_read(  # noqa: E731
        ctypes.byref(c), s, n, k, FAKE, dt, 1024, 128, 1024, 128, None, None)
    assert read(n=0, k=None) == kvr.KVR_OK
    assert read(k=None) == kvr.KVR_E_NULL and read(s=None) == kvr.KVR_E_NULL
    assert read(n=-1) == kvr.KVR_E_SIZE and read(dt=-1) == kvr.KVR_E_LAYOUT


def test_rotary_refusals(lib):
    def call(x=FAKE, out=FAKE, dt=0, n=4, h=8, d=128, st=(1024, 128, 1024, 128), pos=FAKE, table=FAKE, n_pos=16,
             rot=128, flags=0):
        return lib.kvr_rotary(x, out, dt, n, h, d, *st, pos, table, n_pos, rot, flags, None, None)

    assert call(n=0) == kvr.KVR_OK
    for kw in (dict(x=None), dict(out=None), dict(pos=None), dict(table=None)):
        assert call(**kw) == kvr.KVR_E_NULL
    for kw in (dict(n=-1), dict(h=0), dict(h=1 << 17), dict(d=1), dict(d=5000), dict(n=1 << 30), dict(rot=0),
               dict(rot=7), dict(rot=130), dict(n_pos=0), dict(d=512, rot=258)):
        assert call(**kw) == kvr.KVR_E_SIZE
    for kw in (dict(dt=7), dict(st=(-1, 128, 1024, 128)), dict(x=ctypes.c_void_p(0x1001)),
               dict(table=ctypes.c_void_p(0x1001))):
        assert call(**kw) == kvr.KVR_E_LAYOUT
    assert call(flags=8) == kvr.KVR_E_METHOD


def test_rotary_table_refusals(lib):
    def call(rot=128, n=4, table=FAKE, **kw):
        r = kvr.kvr_rope(theta=1e4, factor=4.0, low=1.0, high=32.0, trained_len=4096.0, magnitude=1.0, kind=4)
        for k, v in kw.items():
            setattr(r, k, v)
        return lib.kvr_rotary_table(ctypes.byref(r), rot, n, table, None)

    assert call(n=0) == kvr.KVR_OK
    assert call(table=None) == kvr.KVR_E_NULL
    assert lib.kvr_rotary_table(None, 128, 4, FAKE, None) == kvr.KVR_E_NULL
    for kw in (dict(rot=0), dict(rot=5), dict(rot=258), dict(n=-1), dict(n=1 << 36), dict(rot=2, kind=2)):
        assert call(**kw) == kvr.KVR_E_SIZE
    for kw in (dict(theta=1.0), dict(theta=math.nan), dict(theta=math.inf), dict(factor=0.5), dict(factor=math.nan),
               dict(low=0.0), dict(high=1.0), dict(high=math.inf), dict(trained_len=0.0), dict(magnitude=0.0),
               dict(magnitude=math.inf)):
        assert call(**kw) == kvr.KVR_E_GRID
    assert call(kind=5) == kvr.KVR_E_METHOD and call(kind=-1) == kvr.KVR_E_METHOD


def _attend(lib, c, dt=0, h=32, mask=None, words=0, scale=0.1, ws=FAKE, nbytes=1 << 40, out=FAKE, st=(4096, 128, 4096, 128),
            q=FAKE, sz=None, **kw):
    s = kvr.kvr_sequences(d_cu_q=0x1000, d_kv_len=0x1000, d_pages=0x1000, pages_stride=8, max_pages=8,
                          n_queries=12, n_seqs=4, max_q=3, max_kv=128)
    for k, v in kw.items():
        setattr(s, k, v)
    n = ctypes.c_size_t(nbytes) if sz is None else sz
    return lib.kvr_tree_attention(ctypes.byref(c), ctypes.byref(s), q, dt, h, st[0], st[1], mask, words, scale, out,
                                  st[2], st[3], None, None, ws, ctypes.byref(n), None)


def test_attention_refusals(lib):
    c = _cache()
    assert _attend(lib, c, n_seqs=0) == kvr.KVR_OK
    assert _attend(lib, c, n_queries=0) == kvr.KVR_OK
    for kw in (dict(q=None), dict(out=None), dict(d_cu_q=None), dict(d_kv_len=None), dict(d_pages=None)):
        assert _attend(lib, c, **kw) == kvr.KVR_E_NULL
    for kw in (dict(h=31), dict(h=4), dict(n_seqs=-1), dict(n_seqs=4097), dict(max_q=0), dict(max_kv=0),
               dict(max_kv=(1 << 30) + 1), dict(n_queries=-1), dict(max_pages=-1), dict(max_q=1 << 20),
               dict(mask=FAKE, words=0), dict(mask=FAKE, words=1, max_q=65)):
        assert _attend(lib, c, **kw) == kvr.KVR_E_SIZE, kw
    for kw in (dict(dt=2), dict(dt=5), dict(st=(4095, 128, 4096, 128)), dict(st=(4096, 128, 4096, -8)),
               dict(out=ctypes.c_void_p(0x1008))):
        assert _attend(lib, c, **kw) == kvr.KVR_E_LAYOUT, kw
    assert _attend(lib, _cache(kvr.KVR_KV_BF16, token_stride=256), dt=1) == kvr.KVR_E_LAYOUT
    assert _attend(lib, _cache(kvr.KVR_KV_FP16, token_stride=256), dt=0) == kvr.KVR_E_LAYOUT
    for scale in (math.nan, math.inf, -math.inf):
        assert _attend(lib, c, scale=scale) == kvr.KVR_E_GRID


def test_attention_workspace(lib):
    c = _cache()
    sz = ctypes.c_size_t(0)
    assert _attend(lib, c, ws=None, sz=sz) == kvr.KVR_OK
    assert sz.value == 0                              # short sequences are not cut
    assert _attend(lib, c, ws=None, sz=sz, max_kv=100000, max_q=1) == kvr.KVR_OK
    one = sz.value
    assert one > 0
    assert _attend(lib, c, ws=ctypes.c_void_p(0x1010), max_kv=100000, max_q=1) == kvr.KVR_E_WORKSPACE
    assert _attend(lib, c, nbytes=one - 1, max_kv=100000, max_q=1) == kvr.KVR_E_WORKSPACE
    assert _attend(lib, c, nbytes=one, max_kv=100000, max_q=1, out=None) == kvr.KVR_E_NULL
    # bounded by the parts that fill the GPU, not by the longest sequence
    assert _attend(lib, c, ws=None, sz=sz, max_kv=1 << 30, max_q=1) == kvr.KVR_OK
    assert sz.value == one < (64 << 20)


def test_kv_bytes_per_token():
    """The cost model's KV bytes per token of the 16-bit geometries, and of the formats
    that a row of 128 elements takes 132 and 68 bytes in."""
    assert kvr.kv_bytes_per_token(kvr.KVR_KV_FP16, 32, 8, 128) == 131072
    assert kvr.kv_bytes_per_token(kvr.KVR_KV_BF16, 80, 8, 128) == 327680
    assert kvr.kv_bytes_per_token(kvr.KVR_KV_FP8, 32, 8, 128) == 32 * 8 * 2 * 132
    assert kvr.kv_bytes_per_token(kvr.KVR_KV_FP4, 32, 8, 128) == 32 * 8 * 2 * 68


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_reference_quantisation_is_nearest(fmt):
    """No other code of the block's scale is closer, no smaller scale would do, and packing
    is undone by unpacking."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((40, 64)) * np.exp2(rng.integers(-30, 30, (40, 1)))
    codes, scale = ref.quantise(x, fmt)
    back = ref.dequantise(codes, scale, fmt)
    grid = ref.values_of(fmt)
    grid = np.sort(grid[np.isfinite(grid)])
    s = np.repeat(np.ldexp(1.0, scale.astype(int) - 127), 32, -1)
    best = np.abs((x / s)[..., None] - grid).min(-1) * s
    assert np.array_equal(np.abs(back - x), best)
    amax = np.abs(x).reshape(40, 2, 32).max(-1)
    k = scale.astype(int) - 127
    assert (amax <= np.ldexp(ref.LARGEST[fmt], k)).all() and (amax > np.ldexp(ref.LARGEST[fmt], k - 1)).all()
    assert np.array_equal(ref.unpack(ref.pack(codes, fmt), fmt), codes)


def test_reference_rotation_and_attention():
    """A rotation keeps each pair's length and its adjoint undoes it; attention with one
    visible token is that token's value, and hidden tokens do not matter."""
    rng = np.random.default_rng(4)
    a = rng.uniform(0, 6, (5, 8))
    x = rng.standard_normal((5, 3, 20))
    for il in (False, True):
        y = ref.rotate(x, np.cos(a), np.sin(a), il)
        assert np.allclose(ref.rotate(y, np.cos(a), np.sin(a), il, True), x, atol=1e-14)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1), atol=1e-13)
        g, eps = rng.standard_normal(x.shape), 1e-6
        d = rng.standard_normal(x.shape)
        diff = ((ref.rotate(x + eps * d, np.cos(a), np.sin(a), il) - y) / eps * g).sum()
        assert np.isclose(diff, (ref.rotate(g, np.cos(a), np.sin(a), il, True) * d).sum(), rtol=1e-6)
    q, k, v = (rng.standard_normal((n, 16)) for n in (2, 7, 7))
    seen = np.zeros((2, 7), bool)
    seen[0, 3] = True
    k[5], v[5] = np.nan, np.inf
    out, lse, _, _ = ref.attention(q, k, v, seen, 0.25)
    assert np.allclose(out[0], v[3]) and np.isclose(lse[0], 0.25 * q[0] @ k[3])
    assert (out[1] == 0).all() and lse[1] == -np.inf
