"""Gradients: kvr_rotary's through autograd, against the formula and differences; and the
refusal of tensors whose gradients the other calls would lose."""
import numpy as np
import pytest

from tests import kv_reference as ref
from tests.test_gpu_kv_cache import EPS16, _np, _randn, _table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


@pytest.mark.parametrize("adjoint", [False, True])
@pytest.mark.parametrize("il", [False, True])
@pytest.mark.parametrize("dtype,tokens,heads,dim,rot", [("fp32", 29, 3, 64, 48), ("bf16", 130, 8, 128, 128),
                                                        ("fp16", 1, 1, 34, 10)])
def test_rotary(kvr, dtype, tokens, heads, dim, rot, il, adjoint):
    import torch
    table = _table(5, 31, rot)
    pos = torch.from_numpy(np.random.default_rng(6).integers(0, 31, tokens)).int().cuda()
    wide = _randn(7, (tokens, heads + 2, dim), dtype).requires_grad_()
    x = wide[:, 1:heads + 1]                      # part of a projection
    g = _randn(8, (tokens, heads, dim), dtype)
    y = kvr.kvr_rotary(x, pos, table, interleaved=il, adjoint=adjoint)
    assert y.requires_grad and torch.equal(y, kvr.kvr_rotary(x.detach(), pos, table, interleaved=il, adjoint=adjoint))
    y.backward(g)
    rows = _np(table)[pos.cpu().numpy()]
    want = ref.rotate(_np(g), rows[:, 0], rows[:, 1], il, not adjoint)
    # two products and a sum in 32 bits, then the output's rounding (as the forward's)
    tol = 3 * 2.0 ** -24 * 2 * np.abs(_np(g)).max() + EPS16[dtype] * np.abs(want) * (1 + 1e-6) + (
        2.0 ** -25 if dtype == "fp16" else 0)
    assert (np.abs(_np(wide.grad[:, 1:heads + 1]) - want) <= tol).all()
    assert int(wide.grad[:, 0].count_nonzero()) == 0 and int(wide.grad[:, -1].count_nonzero()) == 0
    if dtype == "fp32":   # <g, f(x + d) - f(x)> = <f'(g), d>: f is linear
        d = _randn(9, (tokens, heads, dim), dtype)
        with torch.no_grad():
            f = [kvr.kvr_rotary(t, pos, table, interleaved=il, adjoint=adjoint).double() for t in (x + d, x)]
        lhs = (g.double() * (f[0] - f[1])).sum(-1)
        rhs = (wide.grad[:, 1:heads + 1].double() * d.double()).sum(-1)
        assert float((lhs - rhs).abs().max()) <= 64 * 8 * 2.0 ** -24 * 100   # 64 terms of a few roundings


def test_rotary_of_expanded_and_second_gradients(kvr):
    import torch
    table, pos = _table(5, 31, 32), torch.arange(12, device="cuda").int()
    x = _randn(1, (12, 2, 64), "fp32").requires_grad_()
    kvr.kvr_rotary(x, pos, table).sum().backward()          # a gradient of strides 0
    want = kvr.kvr_rotary(torch.ones_like(x), pos, table, adjoint=True)
    assert torch.equal(x.grad, want)
    y = kvr.kvr_rotary(x, pos, table)
    g, = torch.autograd.grad((y * y).sum(), x, create_graph=True)     # 2 x but for rounding
    z, = torch.autograd.grad(g.sum(), x)
    assert float((g - 2 * x).abs().max()) <= 64 * 2.0 ** -24 * float(x.abs().max())
    assert float((z - 2).abs().max()) <= 64 * 2.0 ** -24
    with torch.no_grad():
        assert not kvr.kvr_rotary(x, pos, table).requires_grad
        assert kvr.kvr_rotary(x, pos, table, out=torch.empty_like(x)).shape == x.shape
    with pytest.raises(ValueError, match="out"):
        kvr.kvr_rotary(x, pos, table, out=torch.empty_like(x))


def test_rotary_gradient_domain(kvr):
    """A bad position is reported going forward, with autograd as without."""
    import torch
    table, pos = _table(5, 7, 32), torch.tensor([0, 7], device="cuda").int()
    x = _randn(1, (2, 2, 64), "fp32").requires_grad_()
    with pytest.raises(kvr.KvrError) as e:
        kvr.kvr_rotary(x, pos, table)
    assert e.value.code == kvr.KVR_E_DOMAIN
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = kvr.kvr_rotary(x, pos, table, status=status, check=False)
    assert int(status.item()) == kvr.KVR_E_DOMAIN
    y.sum().backward()
    assert x.grad.shape == x.shape


def test_lost_gradients_are_refused(kvr):
    import torch
    cache = kvr.KvCache.allocate(kvr.KVR_KV_BF16, 4, 2, 16, 64)
    x = _randn(1, (5, 2, 64), "bf16")
    slots, pos = torch.arange(5, device="cuda"), torch.arange(5, device="cuda").int()
    table = _table(2, 8, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    att = (torch.tensor([0, 2], **i32), torch.tensor([5], **i32), torch.zeros(1, 1, **i32), 2, 5)
    q = _randn(3, (2, 4, 64), "bf16")
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    calls = [lambda t: kvr.kvr_cache_write(cache, t(x), x, slots), lambda t: kvr.kvr_cache_write(cache, x, t(x), slots),
             lambda t: kvr.kvr_cache_write(cache, x, x, slots, pos, t(table)),
             lambda t: kvr.kvr_cache_read(cache, slots, out=(t(x), t(x))),
             lambda t: kvr.kvr_tree_attention(cache, t(q), *att),
             lambda t: kvr.kvr_tree_attention(cache, q, *att, out=t(q)),
             lambda t: kvr.kvr_rotary(x, pos, t(table)), lambda t: kvr.kvr_rotary(x, pos, table, out=t(x)),
             lambda t: kvr.kvr_tree_attention(kvr.KvCache(cache.k, t(cache.v)), q, *att)]
    for call in calls:
        call(lambda t: t.clone())
        with pytest.raises(ValueError, match="requires gradients"):
            call(leaf)
        with torch.no_grad():
            call(leaf)
        with torch.inference_mode():
            call(leaf)


def test_written_tensors_are_noticed(kvr):
    """A tensor that autograd has saved and a call then writes: backward says so, as after
    torch's own operations in place."""
    import torch
    cache = kvr.KvCache.allocate(kvr.KVR_KV_BF16, 4, 2, 16, 64)
    x = _randn(1, (5, 2, 64), "bf16")
    slots, pos = torch.arange(5, device="cuda"), torch.arange(5, device="cuda").int()
    table = _table(2, 8, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    att = (torch.tensor([0, 2], **i32), torch.tensor([5], **i32), torch.zeros(1, 1, **i32), 2, 5)
    q, out = _randn(3, (2, 4, 64), "bf16"), torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    a, b, y = (torch.empty_like(x) for _ in range(3))
    writes = [(cache.k, lambda: kvr.kvr_cache_write(cache, x, x, slots)),
              (cache.v, lambda: kvr.kvr_cache_write(cache, x, x, slots, check=False)),
              (a, lambda: kvr.kvr_cache_read(cache, slots, out=(a, b))),
              (b, lambda: kvr.kvr_cache_read(cache, slots, out=(a, b))),
              (y, lambda: kvr.kvr_rotary(x, pos, table, out=y)),
              (out, lambda: kvr.kvr_tree_attention(cache, q, *att, out=out))]
    for t, write in writes:
        w = torch.ones_like(t, requires_grad=True)
        loss = (w * t).sum()          # saves t
        kvr.kvr_cache_read(cache, slots)
        kvr.kvr_tree_attention(cache, q, *att)
        loss.backward(retain_graph=True)
        write()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    quant = kvr.KvCache.allocate(kvr.KVR_KV_FP4, 4, 2, 16, 64)
    before = [t._version for t in quant.tensors]
    kvr.kvr_cache_write(quant, x, x, slots)
    assert [t._version for t in quant.tensors] == [n + 1 for n in before]
    with torch.inference_mode():
        kvr.kvr_cache_write(quant, x, x, slots)
        own = torch.empty_like(x)
    kvr.kvr_rotary(x, pos, table, out=own)      # has no version
