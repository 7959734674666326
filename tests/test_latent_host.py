"""C-ABI checks of the latent cache's and the pages' entry points that need no GPU: bad
arguments are refused with the documented codes before the device is touched, workspaces are
sized, empty calls succeed."""
import ctypes
import os

import pytest

import paper_2608_30830_amd as kvr

FAKE = ctypes.c_void_p(0x1000)   # never dereferenced
ODD = ctypes.c_void_p(0x1008)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kvr.LIB_PATH):
        from paper_2608_30830_amd import build
        build.build()
    return kvr.load_library()


def _cache(fmt=None, **kw):
    c = kvr.kvr_latent_cache(data=0x1000, scale=0x2000, page_stride=16 * 576, token_stride=576,
                             scale_page_stride=16 * 18, scale_token_stride=18, n_pages=10, page_size=16,
                             rank=512, rot=64, format=kvr.KVR_KV_FP8 if fmt is None else fmt)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _write(lib, c, latent=FAKE, key=FAKE, dt=0, n=4, st=(576, 576), norm=None, eps=1e-6, slots=FAKE, pos=None,
           table=None, n_pos=0, rot=0, flags=0):
    return lib.kvr_latent_write(None if c is None else ctypes.byref(c), latent, key, dt, n, *st, norm, eps, slots,
                                pos, table, n_pos, rot, flags, None, None)


def _read(lib, c, slots=FAKE, n=4, out=FAKE, dt=0, st=576):
    return lib.kvr_latent_read(None if c is None else ctypes.byref(c), slots, n, out, dt, st, None, None)


def _attend(lib, c, q=FAKE, dt=0, heads=16, st=(16 * 576, 576, 16 * 512, 512), mask=None, words=0, scale=0.1, out=FAKE,
            ws=FAKE, size=1 << 40, none=(), **kw):
    s = kvr.kvr_sequences(d_cu_q=0x1000, d_kv_len=0x1000, d_pages=0x1000, pages_stride=10, max_pages=10, n_queries=4,
                          n_seqs=2, max_q=3, max_kv=9000)
    for k, v in kw.items():
        setattr(s, k, v)
    need = ctypes.c_size_t(size)
    rc = lib.kvr_latent_attention(None if c is None else ctypes.byref(c), None if "seqs" in none else ctypes.byref(s), q,
                                  dt, heads, st[0], st[1], mask, words, scale, out, st[2], st[3], None, None, ws,
                                  None if "size" in none else ctypes.byref(need), None)
    return (rc, need.value) if ws is None else rc


BAD_CACHES = [
    (dict(data=None), kvr.KVR_E_NULL), (dict(scale=None), kvr.KVR_E_NULL), (dict(format=3), kvr.KVR_E_LAYOUT),
    (dict(format=-1), kvr.KVR_E_LAYOUT), (dict(n_pages=0), kvr.KVR_E_SIZE), (dict(n_pages=1 << 31), kvr.KVR_E_SIZE),
    (dict(page_size=8), kvr.KVR_E_LAYOUT), (dict(page_size=48), kvr.KVR_E_LAYOUT),
    (dict(page_size=1 << 16), kvr.KVR_E_LAYOUT), (dict(rank=128), kvr.KVR_E_LAYOUT), (dict(rank=1024), kvr.KVR_E_LAYOUT),
    (dict(rot=0), kvr.KVR_E_LAYOUT), (dict(rot=128), kvr.KVR_E_LAYOUT), (dict(data=0x1008), kvr.KVR_E_LAYOUT),
    (dict(token_stride=584), kvr.KVR_E_LAYOUT), (dict(page_stride=-16), kvr.KVR_E_LAYOUT),
    (dict(token_stride=1 << 27), kvr.KVR_E_LAYOUT), (dict(scale_token_stride=-1), kvr.KVR_E_LAYOUT),
    (dict(scale_page_stride=-1), kvr.KVR_E_LAYOUT),
]


@pytest.mark.parametrize("kw,code", BAD_CACHES, ids=lambda x: str(x))
def test_bad_caches(lib, kw, code):
    c = _cache(**kw)
    assert _write(lib, c) == code and _read(lib, c) == code and _attend(lib, c) == code
    assert _attend(lib, c, ws=None)[0] == code


def test_write_and_read_refusals(lib):
    c = _cache()
    assert _write(lib, None) == kvr.KVR_E_NULL and _read(lib, None) == kvr.KVR_E_NULL
    assert _write(lib, c, n=0) == kvr.KVR_OK and _read(lib, c, n=0, out=None, slots=None) == kvr.KVR_OK
    assert _write(lib, c, n=0, latent=None, key=None, slots=None) == kvr.KVR_OK
    for n in (-1, 1 << 31):
        assert _write(lib, c, n=n) == kvr.KVR_E_SIZE and _read(lib, c, n=n) == kvr.KVR_E_SIZE
    for dt in (-1, 3):
        assert _write(lib, c, dt=dt) == kvr.KVR_E_LAYOUT and _read(lib, c, dt=dt) == kvr.KVR_E_LAYOUT
    for kw in (dict(latent=None), dict(key=None), dict(slots=None)):
        assert _write(lib, c, **kw) == kvr.KVR_E_NULL
    assert _read(lib, c, slots=None) == kvr.KVR_E_NULL and _read(lib, c, out=None) == kvr.KVR_E_NULL
    for kw in (dict(latent=ODD), dict(key=ODD), dict(st=(572, 576)), dict(st=(576, -8)), dict(norm=ODD)):
        assert _write(lib, c, **kw) == kvr.KVR_E_LAYOUT
    assert _read(lib, c, out=ODD) == kvr.KVR_E_LAYOUT and _read(lib, c, st=570) == kvr.KVR_E_LAYOUT
    for eps in (-1e-6, float("nan"), float("inf")):
        assert _write(lib, c, norm=FAKE, eps=eps) == kvr.KVR_E_GRID
        assert _write(lib, c, n=0, eps=eps) == kvr.KVR_OK   # no norm, no matter
    assert _write(lib, c, table=FAKE, n_pos=9, rot=64) == kvr.KVR_E_NULL   # no positions
    for rot in (0, 3, 66, -2):
        assert _write(lib, c, pos=FAKE, table=FAKE, n_pos=9, rot=rot) == kvr.KVR_E_SIZE
    assert _write(lib, c, pos=FAKE, table=FAKE, n_pos=0, rot=64) == kvr.KVR_E_SIZE
    assert _write(lib, c, pos=FAKE, table=ctypes.c_void_p(0x1002), n_pos=9, rot=64) == kvr.KVR_E_LAYOUT
    assert _write(lib, c, pos=FAKE, table=FAKE, n_pos=9, rot=64, flags=4) == kvr.KVR_E_METHOD


def test_attention_refusals(lib):
    c = _cache()
    rc, need = _attend(lib, c, ws=None)
    assert rc == kvr.KVR_OK and need > 0
    assert _attend(lib, c, ws=None, q=None, out=None, d_cu_q=None, d_kv_len=None, d_pages=None) == (kvr.KVR_OK, need)
    assert _attend(lib, c, ws=None, max_kv=100) == (kvr.KVR_OK, 0)   # nothing is cut
    assert _attend(lib, c, size=need - 1) == kvr.KVR_E_WORKSPACE
    assert _attend(lib, c, ws=ctypes.c_void_p(0x1010)) == kvr.KVR_E_WORKSPACE
    assert _attend(lib, None) == kvr.KVR_E_NULL
    for none in ("seqs", "size"):
        assert _attend(lib, c, none=(none,)) == kvr.KVR_E_NULL
    for kw in (dict(q=None), dict(out=None), dict(d_cu_q=None), dict(d_kv_len=None), dict(d_pages=None)):
        assert _attend(lib, c, **kw) == kvr.KVR_E_NULL
    assert _attend(lib, c, n_seqs=0) == kvr.KVR_OK and _attend(lib, c, n_queries=0) == kvr.KVR_OK
    for kw in (dict(n_seqs=-1), dict(n_seqs=4097), dict(max_q=0), dict(max_kv=0), dict(max_kv=(1 << 30) + 1),
               dict(n_queries=-1), dict(n_queries=1 << 31), dict(max_pages=-1), dict(pages_stride=-1), dict(heads=0),
               dict(max_q=1 << 21), dict(mask=FAKE, words=0), dict(mask=FAKE, words=1, max_q=65)):
        assert _attend(lib, c, **kw) == kvr.KVR_E_SIZE, kw
    for fmt, wrong in ((kvr.KVR_KV_FP8, 1), (kvr.KVR_KV_FP8, 2), (kvr.KVR_KV_BF16, 1), (kvr.KVR_KV_FP16, 0)):
        assert _attend(lib, _cache(fmt), dt=wrong) == kvr.KVR_E_LAYOUT
    for kw in (dict(q=ODD), dict(out=ODD), dict(st=(16 * 576 + 4, 576, 8192, 512)), dict(st=(9216, 576, 8192, -512))):
        assert _attend(lib, c, **kw) == kvr.KVR_E_LAYOUT
    for scale in (float("nan"), float("inf")):
        assert _attend(lib, c, scale=scale) == kvr.KVR_E_GRID


def _prompt(lib, dt=0, q=FAKE, k=FAKE, r=FAKE, v=FAKE, out=FAKE, scale=0.1, ws=FAKE, size=1 << 40, none=(),
            st=(4 * 192, 192, 512, 128, 64, 512, 128, 512, 128), **kw):
    p = kvr.kvr_prompt(d_cu_q=0x1000, d_cu_k=0x1000, n_queries=10, n_keys=5000, n_seqs=2, max_q=5, max_k=4000, n_q_heads=4,
                       n_kv_heads=4, nope=128, rot=64, causal=1)
    for name, value in kw.items():
        setattr(p, name, value)
    need = ctypes.c_size_t(size)
    rc = lib.kvr_latent_prompt(None if "prompt" in none else ctypes.byref(p), q, dt, st[0], st[1], k, st[2], st[3], r, st[4],
                               v, st[5], st[6], scale, out, st[7], st[8], None, None, ws,
                               None if "size" in none else ctypes.byref(need), None)
    return (rc, need.value) if ws is None else rc


def test_prompt_refusals(lib):
    rc, need = _prompt(lib, ws=None)
    assert rc == kvr.KVR_OK and need > 0                               # few queries, many keys
    assert _prompt(lib, ws=None, max_k=64) == (kvr.KVR_OK, 0)          # nothing to cut
    assert _prompt(lib, size=need - 1) == kvr.KVR_E_WORKSPACE
    assert _prompt(lib, ws=ctypes.c_void_p(0x1010)) == kvr.KVR_E_WORKSPACE
    for none in ("prompt", "size"):
        assert _prompt(lib, none=(none,)) == kvr.KVR_E_NULL
    for kw in (dict(q=None), dict(k=None), dict(r=None), dict(v=None), dict(out=None), dict(d_cu_q=None), dict(d_cu_k=None)):
        assert _prompt(lib, **kw) == kvr.KVR_E_NULL, kw
    assert _prompt(lib, n_seqs=0) == kvr.KVR_OK and _prompt(lib, n_queries=0, q=None) == kvr.KVR_OK
    for kw in (dict(n_seqs=-1), dict(n_seqs=4097), dict(max_q=0), dict(max_k=0), dict(max_k=(1 << 30) + 1),
               dict(n_queries=-1), dict(n_queries=1 << 31), dict(n_keys=-1), dict(n_keys=1 << 31), dict(n_q_heads=0),
               dict(n_kv_heads=0), dict(n_kv_heads=3), dict(n_q_heads=2), dict(n_kv_heads=2048, n_q_heads=2048),
               dict(n_q_heads=4100), dict(max_q=1 << 29), dict(n_queries=(1 << 31) - 1, n_q_heads=64)):
        assert _prompt(lib, **kw) == kvr.KVR_E_SIZE, kw
    for kw in (dict(dt=2), dict(nope=96), dict(nope=256), dict(rot=0), dict(rot=128), dict(q=ODD), dict(k=ODD), dict(r=ODD),
               dict(v=ODD), dict(out=ODD), dict(st=(768, 188, 512, 128, 64, 512, 128, 512, 128)),
               dict(st=(768, 192, 512, 128, 60, 512, 128, 512, 128)), dict(st=(768, 192, 512, 128, 64, -512, 128, 512, 128)),
               dict(st=(768, 192, (1 << 24) + 8, 128, 64, 512, 128, 512, 128))):
        assert _prompt(lib, **kw) == kvr.KVR_E_LAYOUT, kw
    for causal in (-1, 2):
        assert _prompt(lib, causal=causal) == kvr.KVR_E_METHOD
    assert _prompt(lib, scale=float("nan")) == kvr.KVR_E_GRID


def _pool(**kw):
    p = kvr.kvr_page_pool(d_refs=0x1000, d_pages=0x1000, d_kv_len=0x1000, n_pages=100, pages_stride=8, max_pages=8,
                          n_seqs=3, page_size=16)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _calls(lib, p, ws=FAKE, size=1 << 40, most=100):
    """fork, resize and compact of a pool, with everything else in order."""
    n = ctypes.c_size_t(size)
    p = None if p is None else ctypes.byref(p)
    return (lib.kvr_pages_fork(p, FAKE, None, None), lib.kvr_pages_resize(p, FAKE, FAKE, None, ws, ctypes.byref(n), None),
            lib.kvr_pages_compact(p, FAKE, most, FAKE, None, ws, ctypes.byref(n), None))


def test_pool_refusals(lib):
    assert set(_calls(lib, None)) == {kvr.KVR_E_NULL}
    for kw in (dict(n_pages=0), dict(n_pages=(1 << 30) + 1), dict(n_seqs=-1), dict(n_seqs=65537), dict(max_pages=-1),
               dict(max_pages=(1 << 24) + 1, pages_stride=1 << 25), dict(pages_stride=-1)):
        assert set(_calls(lib, _pool(**kw))) == {kvr.KVR_E_SIZE}, kw
    for kw in (dict(page_size=8), dict(page_size=24), dict(page_size=1 << 16), dict(pages_stride=7), dict(pages_stride=0)):
        assert set(_calls(lib, _pool(**kw))) == {kvr.KVR_E_LAYOUT}, kw
    for kw in (dict(d_refs=None), dict(d_pages=None), dict(d_kv_len=None)):
        assert set(_calls(lib, _pool(**kw))) == {kvr.KVR_E_NULL}, kw
    p = ctypes.byref(_pool())
    n = ctypes.c_size_t(1 << 40)
    assert lib.kvr_pages_fork(p, None, None, None) == kvr.KVR_E_NULL
    assert lib.kvr_pages_resize(p, None, FAKE, None, FAKE, ctypes.byref(n), None) == kvr.KVR_E_NULL
    assert lib.kvr_pages_resize(p, FAKE, None, None, FAKE, ctypes.byref(n), None) == kvr.KVR_E_NULL
    assert lib.kvr_pages_resize(p, FAKE, FAKE, None, FAKE, None, None) == kvr.KVR_E_NULL
    assert lib.kvr_pages_compact(p, None, 5, FAKE, None, FAKE, ctypes.byref(n), None) == kvr.KVR_E_NULL
    assert lib.kvr_pages_compact(p, FAKE, 5, None, None, FAKE, ctypes.byref(n), None) == kvr.KVR_E_NULL
    for most in (-1, 101):
        assert _calls(lib, _pool(), most=most)[2] == kvr.KVR_E_SIZE
    assert lib.kvr_pages_fork(ctypes.byref(_pool(n_seqs=0)), None, None, None) == kvr.KVR_OK


def test_pool_workspaces(lib):
    for call in (lambda ws, n: lib.kvr_pages_resize(ctypes.byref(_pool()), FAKE, FAKE, None, ws, ctypes.byref(n), None),
                 lambda ws, n: lib.kvr_pages_compact(ctypes.byref(_pool()), FAKE, 5, FAKE, None, ws, ctypes.byref(n), None)):
        n = ctypes.c_size_t(0)
        assert call(None, n) == kvr.KVR_OK and n.value > 0
        assert call(FAKE, ctypes.c_size_t(n.value - 1)) == kvr.KVR_E_WORKSPACE
        assert call(ctypes.c_void_p(0x1010), ctypes.c_size_t(1 << 40)) == kvr.KVR_E_WORKSPACE


def test_copy_refusals(lib):
    def call(n=1, pages=10, pairs=FAKE, count=4, buffers=True, **kw):
        b = (kvr.kvr_page_buffer * 2)()
        for x in b:
            x.data, x.page_stride, x.run_bytes, x.outer, x.inner = 0x1000, 4096, 4096, 1, 1
        for k, v in kw.items():
            setattr(b[0], k, v)
        return lib.kvr_pages_copy(b if buffers else None, n, pages, pairs, count, None, None)

    assert call(n=0) == kvr.KVR_OK and call(count=0) == kvr.KVR_OK and call(n=0, buffers=False) == kvr.KVR_OK
    for kw in (dict(n=-1), dict(n=65537), dict(pages=0), dict(pages=1 << 31), dict(count=-1), dict(count=(1 << 30) + 1),
               dict(outer=0), dict(inner=0), dict(run_bytes=0), dict(run_bytes=1 << 41),
               dict(outer=1 << 20, inner=1 << 20, run_bytes=2)):
        assert call(**kw) == kvr.KVR_E_SIZE, kw
    for kw in (dict(pairs=None), dict(buffers=False), dict(data=None)):
        assert call(**kw) == kvr.KVR_E_NULL, kw
    for kw in (dict(page_stride=-1), dict(outer_stride=-1), dict(inner_stride=-16)):
        assert call(**kw) == kvr.KVR_E_LAYOUT, kw


def test_bytes_per_token():
    assert kvr.latent_bytes_per_token(kvr.KVR_KV_BF16, 3, 512, 64) == 3 * 1152
    assert kvr.latent_bytes_per_token(kvr.KVR_KV_FP8, 2, 256, 32) == 2 * (288 + 9)
