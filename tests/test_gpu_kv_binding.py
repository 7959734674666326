"""What the tensor binding of the cache's entry points refuses, and what it returns."""
import pytest
import torch

import paper_2608_30830_amd as kvr

pytestmark = pytest.mark.gpu


def _setup():
    cache = kvr.KvCache.allocate(kvr.KVR_KV_FP8, 4, 2, 16, 64)
    x = torch.randn(5, 2, 64, device="cuda").bfloat16()
    slots = torch.arange(5, device="cuda")
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    table = kvr.kvr_rotary_table(64, 8)
    att = dict(q=torch.randn(2, 4, 64, device="cuda").bfloat16(),
               cu_q=torch.tensor([0, 2], dtype=torch.int32, device="cuda"),
               kv_len=torch.tensor([5], dtype=torch.int32, device="cuda"),
               page_table=torch.zeros(1, 1, dtype=torch.int32, device="cuda"), max_q=2, max_kv=5)
    return cache, x, slots, pos, table, att


def test_rotary_refuses():
    _, x, _, pos, table, _ = _setup()
    call = lambda **k: kvr.kvr_rotary(**{**dict(x=x, positions=pos, table=table, check=False), **k})  # noqa: E731
    for bad in (dict(x=x.cpu()), dict(x=x[0]), dict(x=x.transpose(1, 2)), dict(x=x.double()),
                dict(positions=pos.long()), dict(positions=pos[:4]), dict(positions=pos.cpu()),
                dict(positions=torch.stack([pos, pos], 1)[:, 0]), dict(table=table.double()),
                dict(table=table[:, :1]), dict(table=table[:, :, ::2]), dict(table=table[0]),
                dict(out=x[:4]), dict(out=x.float()), dict(status=torch.zeros(2, dtype=torch.int32, device="cuda")),
                dict(status=torch.zeros(1, device="cuda"))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(x=None), dict(x=3), dict(positions=None), dict(table=[1.0])):
        with pytest.raises(TypeError):
            call(**bad)
    wide = kvr.kvr_rotary_table(128, 8)     # more than the head has
    with pytest.raises(kvr.KvrError) as e:
        call(table=wide)
    assert e.value.code == kvr.KVR_E_SIZE
    assert call(x=x[:0], positions=pos[:0]).shape == (0, 2, 64)
    y = torch.empty_like(x)
    assert call(out=y) is y


def test_cache_refuses():
    cache, x, slots, pos, table, _ = _setup()
    call = lambda **k: kvr.kvr_cache_write(**{**dict(cache=cache, k=x, v=x, slots=slots, check=False), **k})  # noqa: E731
    for bad in (dict(k=x[:4]), dict(v=x[:, :1]), dict(k=x[..., :32]), dict(v=x.half()), dict(k=x.int()),
                dict(slots=slots.int()), dict(slots=slots.cpu()), dict(table=table), dict(positions=pos),
                dict(table=table, positions=pos[:2])):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(kvr.KvrError) as e:   # rows off 16 bytes
        call(k=torch.empty(5, 2, 72, device="cuda", dtype=torch.bfloat16)[..., 4:68])
    assert e.value.code == kvr.KVR_E_LAYOUT
    call()
    read = lambda **k: kvr.kvr_cache_read(**{**dict(cache=cache, slots=slots, check=False), **k})  # noqa: E731
    for bad in (dict(dtype=torch.float64), dict(slots=slots.int()), dict(out=(x, x.float())),
                dict(out=(x, x), dtype=torch.float32), dict(out=(x[:4], x[:4]))):
        with pytest.raises(ValueError):
            read(**bad)
    for dt in (torch.bfloat16, torch.float16, torch.float32):
        k, v = read(dtype=dt)
        assert k.dtype == dt and torch.equal(k, v) and k.is_contiguous()
    k2 = torch.empty_like(x)
    k, v = read(out=(k2, torch.empty_like(x)))
    assert k is k2 and torch.equal(k, v)


def test_attention_refuses():
    cache, x, slots, _, _, att = _setup()
    kvr.kvr_cache_write(cache, x, x, slots)
    call = lambda **k: kvr.kvr_tree_attention(cache, **{**att, "check": False, **k})  # noqa: E731
    mask = torch.tensor([[1], [3]], device="cuda")
    for bad in (dict(q=att["q"].float()[..., :32]), dict(q=att["q"].double()), dict(cu_q=att["cu_q"][:1]),
                dict(kv_len=att["kv_len"].long()), dict(page_table=att["page_table"][0]),
                dict(page_table=att["page_table"].long()), dict(tree_mask=mask[:1]),
                dict(tree_mask=mask.int()), dict(out=att["q"].half()), dict(workspace=mask),
                dict(max_kv=1 << 40)):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(max_q="2"), dict(scale="x"), dict(kv_len=5)):
        with pytest.raises(TypeError):
            call(**bad)
    for bad, code in ((dict(q=att["q"].float()), kvr.KVR_E_LAYOUT), (dict(max_q=0), kvr.KVR_E_SIZE),
                      (dict(q=att["q"][:, :1]), kvr.KVR_E_SIZE), (dict(scale=float("nan")), kvr.KVR_E_GRID)):
        with pytest.raises(kvr.KvrError) as e:
            call(**bad)
        assert e.value.code == code
    out, lse = call(want_lse=True, tree_mask=mask)
    plain = call()      # the tree is a chain here
    assert torch.equal(out, plain) and out.dtype == torch.bfloat16 and lse.shape == (2, 4)
    scaled = call(scale=64 ** -0.5, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert torch.equal(scaled, out)
    on = torch.cuda.Stream()
    on.wait_stream(torch.cuda.current_stream())
    other = call(stream=on)
    on.synchronize()
    assert torch.equal(other, out)
