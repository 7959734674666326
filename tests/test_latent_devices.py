"""The tensors of one call are of one device, for the latent cache's and the pages' calls: what
the binding refuses before it touches memory or a GPU.  (Tensors without memory stand in for a
second GPU's.)"""
import pytest
import torch

import paper_2608_30830_amd as kvr
from tests.test_kv_devices import fast, on  # noqa: F401

I32, I64 = torch.int32, torch.int64


def _cache(on, device=0, scale=0):
    t = on(device, (4, 16, 288), torch.uint8), on(scale, (4, 16, 9), torch.uint8)
    for x in t:
        x.data_ptr = lambda: 0x1000   # never read
    return kvr.LatentCache(t[0], 32, t[1])


def _each(call, names):
    for bad in names:
        with pytest.raises(ValueError, match=f"{bad} must be o.* cuda:0"):
            call(lambda n: int(n == bad))


def test_cache(on):  # noqa: F811
    assert _cache(on).device == torch.device("cuda", 0)
    with pytest.raises(ValueError, match="one device"):
        _cache(on, scale=1)
    rows, scale = on(0, (4, 16, 288), torch.uint8), on(0, (4, 16, 9), torch.uint8)
    for bad in (lambda: kvr.LatentCache(rows, 32), lambda: kvr.LatentCache(rows, 0, scale),
                lambda: kvr.LatentCache(rows, 288, scale), lambda: kvr.LatentCache(on(0, (4, 16, 288), torch.float32), 32),
                lambda: kvr.LatentCache(on(0, (4, 16, 288)), 32, scale),
                lambda: kvr.LatentCache(rows, 32, on(0, (4, 16, 8), torch.uint8)),
                lambda: kvr.LatentCache(rows, 32, on(0, (4, 16, 9), torch.int8)),
                lambda: kvr.LatentCache(on(0, (4, 288)), 32)):
        with pytest.raises(ValueError):
            bad()


def test_write_and_read(fast, on):  # noqa: F811
    def write(d):
        return fast.latent_write(_cache(on).handle, on(d("latent"), (5, 256)), on(d("key"), (5, 32)), on(d("slots"), (5,), I64),
                                 on(d("positions"), (5,), I32), on(d("table"), (8, 2, 16), torch.float32),
                                 on(d("norm_weight"), (256,)), 1e-6, 0, on(d("status"), (1,), I32), (0, d("stream")))

    def read(d):
        return fast.latent_read(_cache(on).handle, on(d("slots"), (5,), I64), None, on(d("out"), (5, 288)),
                                on(d("status"), (1,), I32), (0, d("stream")))

    _each(write, ("latent", "key", "slots", "positions", "table", "norm_weight", "status", "stream"))
    _each(read, ("slots", "out", "status", "stream"))


def test_attention(fast, on):  # noqa: F811
    def call(d):
        return fast.latent_attention(
            _cache(on).handle, on(d("q"), (6, 4, 288)), on(d("cu_q"), (3,), I32), on(d("kv_len"), (2,), I32),
            on(d("page_table"), (2, 3), I32), 3, 40, 0.1, on(d("tree_mask"), (6, 1), I64), False, on(d("out"), (6, 4, 256)),
            on(d("workspace"), (999,), torch.uint8), on(d("status"), (1,), I32), (0, d("stream")))

    _each(call, ("q", "cu_q", "kv_len", "page_table", "tree_mask", "out", "workspace", "status", "stream"))


def test_prompt(fast, on):  # noqa: F811
    def call(d):
        return fast.latent_prompt(
            on(0, (6, 4, 96)), on(d("k"), (9, 2, 64)), on(d("k_rot"), (9, 32)), on(d("v"), (9, 2, 64)), on(d("cu_q"), (3,), I32),
            on(d("cu_k"), (3,), I32), 4, 5, True, None, False, on(d("out"), (6, 4, 64)), on(d("workspace"), (999,), torch.uint8),
            on(d("status"), (1,), I32), (0, d("stream")))

    _each(call, ("k", "k_rot", "v", "cu_q", "cu_k", "out", "workspace", "status", "stream"))


def test_pages(fast, on):  # noqa: F811
    def pool(d):
        return on(0, (9,), I32), on(d("page_table"), (3, 4), I32), on(d("kv_len"), (3,), I32)

    _each(lambda d: fast.pages_fork(*pool(d), on(d("parent"), (3,), I32), 16, on(d("status"), (1,), I32), (0, d("stream"))),
          ("page_table", "kv_len", "parent", "status", "stream"))
    _each(lambda d: fast.pages_resize(*pool(d), on(d("new_len"), (3,), I32), 16, on(d("copies"), (3, 2), I32),
                                      on(d("workspace"), (999,), torch.uint8), on(d("status"), (1,), I32), (0, d("stream"))),
          ("page_table", "kv_len", "new_len", "copies", "workspace", "status", "stream"))
    _each(lambda d: fast.pages_compact(*pool(d), 16, 5, on(d("moves"), (5, 2), I32), on(d("used"), (1,), I32),
                                       on(d("workspace"), (999,), torch.uint8), on(d("status"), (1,), I32), (0, d("stream"))),
          ("page_table", "kv_len", "moves", "used", "workspace", "status", "stream"))
    buffers = kvr.PageBuffers([_cache(on), _cache(on)])
    _each(lambda d: fast.pages_copy(buffers.handle, on(d("pairs"), (3, 2), I32), on(d("status"), (1,), I32), (0, d("stream"))),
          ("pairs", "status", "stream"))
    with pytest.raises(ValueError, match="one device"):
        kvr.PageBuffers([_cache(on), _cache(on, 1, 1)])
    with pytest.raises(ValueError):
        kvr.PageBuffers([])
    with pytest.raises(ValueError):
        kvr.PageBuffers([_cache(on), "cache"])
