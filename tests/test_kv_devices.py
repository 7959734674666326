"""The tensors of one call are of one device: what the binding refuses before it touches
memory or a GPU.  (Tensors without memory stand in for a second GPU's.)"""
import os

import pytest
import torch

import paper_2608_30830_amd as kvr


@pytest.fixture(scope="module")
def fast():
    if not (os.path.exists(kvr.LIB_PATH) and os.path.exists(kvr.kv.BINDING_PATH)):
        from paper_2608_30830_amd import build
        build.build()
    return kvr.kv.load_binding()


@pytest.fixture()
def on():
    """Tensors that say they are on a device, and hold nothing."""
    from torch._subclasses.fake_tensor import FakeTensor, FakeTensorMode
    mode = FakeTensorMode()

    def make(device, shape, dtype=torch.bfloat16):
        meta = torch.empty(shape, dtype=dtype, device="meta")
        return FakeTensor(mode, meta, torch.device("cuda", device))
    return make


def _cache(on, device=0, **other):
    shape = (4, 2, 16, 64)
    parts = dict(k=(device, shape), v=(device, shape), k_scale=(device, shape[:3] + (2,)), v_scale=(device, shape[:3] + (2,)))
    for name, d in other.items():
        parts[name] = (d, parts[name][1])
    t = {n: on(d, s, torch.uint8) for n, (d, s) in parts.items()}
    for x in t.values():
        x.data_ptr = lambda: 0x1000   # never read
    return kvr.KvCache(**t)


def test_stand_ins(on):
    x = on(1, (3, 2, 64))
    assert x.is_cuda and x.device == torch.device("cuda", 1)


@pytest.mark.parametrize("name", ["v", "k_scale", "v_scale"])
def test_cache_of_two_devices(on, name):
    assert _cache(on).device == torch.device("cuda", 0)
    with pytest.raises(ValueError, match="one device"):
        _cache(on, **{name: 1})


def test_rotary(fast, on):
    i32 = torch.int32
    args = lambda d=lambda n: 0: [on(0, (5, 2, 64)), on(d("positions"), (5,), i32),  # noqa: E731
                                  on(d("table"), (8, 2, 32), torch.float32), 0, on(d("out"), (5, 2, 64)),
                                  on(d("status"), (1,), i32), (0, d("stream"))]
    for bad in ("positions", "table", "out", "status", "stream"):
        with pytest.raises(ValueError, match=f"{bad} must be o.* cuda:0"):
            fast.rotary(*args(lambda n: int(n == bad)))


def test_write_and_read(fast, on):
    i32, i64 = torch.int32, torch.int64

    def write(bad):
        d = lambda n: int(n == bad)  # noqa: E731
        return fast.cache_write(_cache(on).handle, on(d("k"), (5, 2, 64)), on(d("v"), (5, 2, 64)), on(d("slots"), (5,), i64),
                                on(d("positions"), (5,), i32), on(d("table"), (8, 2, 32), torch.float32), 0,
                                on(d("status"), (1,), i32), (0, d("stream")))

    def read(bad):
        d = lambda n: int(n == bad)  # noqa: E731
        return fast.cache_read(_cache(on).handle, on(d("slots"), (5,), i64), None, on(d("out k"), (5, 2, 64)),
                               on(d("out v"), (5, 2, 64)), on(d("status"), (1,), i32), (0, d("stream")))

    for call, names in ((write, ("k", "v", "slots", "positions", "table", "status", "stream")),
                        (read, ("slots", "out k", "out v", "status", "stream"))):
        for bad in names:
            with pytest.raises(ValueError, match=f"{bad} must be o.* cuda:0"):
                call(bad)


def test_attention(fast, on):
    i32, i64 = torch.int32, torch.int64

    def call(bad):
        d = lambda n: int(n == bad)  # noqa: E731
        return fast.tree_attention(
            _cache(on).handle, on(d("q"), (6, 4, 64)), on(d("cu_q"), (3,), i32), on(d("kv_len"), (2,), i32),
            on(d("page_table"), (2, 3), i32), 3, 40, on(d("tree_mask"), (6, 1), i64), None, False, on(d("out"), (6, 4, 64)),
            on(d("workspace"), (999,), torch.uint8), on(d("status"), (1,), i32), (0, d("stream")))

    for bad in ("q", "cu_q", "kv_len", "page_table", "tree_mask", "out", "workspace", "status", "stream"):
        with pytest.raises(ValueError, match=f"{bad} must be o.* cuda:0"):
            call(bad)


def test_want_lse_without_a_truth_value(fast, on):
    class Neither:
        def __bool__(self):
            raise RuntimeError("no")

    with pytest.raises(TypeError, match="want_lse"):
        fast.tree_attention(_cache(on).handle, on(0, (6, 4, 64)), on(0, (3,), torch.int32), on(0, (2,), torch.int32),
                            on(0, (2, 3), torch.int32), 3, 40, None, None, Neither(), None, None, None, None)
