"""Attention calls whose first queries decrease: reported, and no part is read that the
plan has no room for."""
import ctypes

import pytest

from tests.test_gpu_kv_attention import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


def _workspace_bytes(kvr, p, n_seqs):
    s = kvr.kvr_sequences(d_cu_q=p.cu_q.data_ptr(), d_kv_len=p.kv_len.data_ptr(), d_pages=p.table.data_ptr(),
                          pages_stride=p.table.shape[1], max_pages=p.table.shape[1], n_queries=p.q.shape[0],
                          n_seqs=n_seqs, max_q=p.max_q, max_kv=p.max_kv)
    n = ctypes.c_size_t(0)
    dtype = kvr.KVR_DT_BF16 if p.dtype == "bf16" else kvr.KVR_DT_FP16
    rc = kvr.load_library().kvr_tree_attention(
        ctypes.byref(p.cache.c), ctypes.byref(s), None, dtype, p.q.shape[1], 0, 0, None, 0, 1.0, None, 0, 0,
        None, None, None, ctypes.byref(n), None)
    assert rc == kvr.KVR_OK
    return n.value


@pytest.mark.parametrize("group", [8, 1])
def test_first_queries_that_decrease(kvr, group):
    """255 sequences of 1,024 tokens with first queries 0, 64, 0, 64, ...: half of them have the
    call's 64 queries, the others fewer than none.  The memory behind the workspace holds NaN."""
    import torch
    p = Problem(kvr, 71, "bf16", "bf16", [1024], [64], 1, group, 128, 64)
    n = 255
    p.cu_q = torch.tensor([0, 64] * 128, dtype=torch.int32, device="cuda")
    p.kv_len = torch.full((n,), 1024, dtype=torch.int32, device="cuda")
    p.table = p.table.repeat(n, 1)
    need = _workspace_bytes(kvr, p, n)
    assert need > 0
    room = torch.full((need + (256 << 20),), 0xFF, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = p.call(workspace=room[:need], status=status, check=False)
    assert int(status.item()) == kvr.KVR_E_DOMAIN
    assert bool((room[need:] == 0xFF).all())
    p.check(out, lse)   # all that are answered have the same tokens
    with pytest.raises(kvr.KvrError) as e:
        p.call()
    assert e.value.code == kvr.KVR_E_DOMAIN
