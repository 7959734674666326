"""How attention's sequences are cut into items, on the host: whatever the lengths in a
call are, no item that is joined lies outside the planned ones, which are what the
workspace holds."""
import os
import subprocess

import numpy as np
import pytest

import paper_2608_30830_amd as kvr
from paper_2608_30830_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
DOMAIN = kvr.KVR_E_DOMAIN


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not os.path.exists(kvr.LIB_PATH):
        build.build()
    lib = os.path.dirname(build.LIB)
    exe = str(tmp_path_factory.mktemp("parts") / "kv_parts")
    subprocess.run([build.HIPCC, "--cuda-host-only", "-x", "hip", "-std=c++17", "-O1", "-I" + build.CSRC,
                    "-I" + os.path.join(build.ROOT, "include"), os.path.join(HERE, "kv_parts.cpp"),
                    "-x", "none", build.LIB, "-Wl,-rpath," + lib, "-o", exe], check=True, capture_output=True,
                   timeout=120)
    return exe


def _run(exe, q_heads, kv_heads, max_q, max_kv, n_queries, cu, kv):
    text = " ".join(str(int(x)) for x in [q_heads, kv_heads, max_q, max_kv, n_queries, len(kv), *cu, *kv])
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=60)
    names = ("status", "planned", "room", "per", "items", "used", "joined", "left")
    return dict(zip(names, map(int, out.stdout.split())))


def test_lengths_that_fit(program):
    rng = np.random.default_rng(1)
    for _ in range(60):
        n = int(np.exp(rng.uniform(0, np.log(300))))
        kv_heads, group = int(rng.choice([1, 2, 8, 32])), int(rng.choice([1, 2, 3, 8, 16]))
        max_q = int(np.exp(rng.uniform(0, np.log(500))))
        nq = rng.integers(0, max_q + 1, n)
        nq[rng.integers(n)] = max_q
        kv = nq + np.exp(rng.uniform(0, np.log(60000), n)).astype(int)
        got = _run(program, kv_heads * group, kv_heads, max_q, int(kv.max()), int(nq.sum()),
                   np.concatenate([[0], np.cumsum(nq)]), kv)
        assert got["status"] == 0 and got["left"] == 0
        assert got["items"] <= got["planned"]
        assert got["room"] == 0 and got["joined"] == 0 or got["room"] == got["planned"]


@pytest.mark.parametrize("kv_heads,group", [(1, 8), (1, 1), (8, 8)])
def test_sequences_that_share_their_queries(program, kv_heads, group):
    """First queries 0, 64, 0, 64, ...: every other sequence has the call's 64 queries, and
    the others fewer than none.  Their items are more than the planned ones."""
    n = 255
    cu = [0, 64] * 128
    got = _run(program, kv_heads * group, kv_heads, 64, 1024, 64, cu, [1024] * n)
    assert got["status"] == DOMAIN
    assert got["room"] == got["planned"] > 0
    assert got["used"] <= got["room"]
    if kv_heads == 1 and group == 8:
        assert got["items"] > got["planned"] and got["left"] > 0 and got["joined"] > 0


def test_any_first_queries(program):
    rng = np.random.default_rng(2)
    over = 0
    for _ in range(60):
        n = int(np.exp(rng.uniform(0, np.log(400))))
        group, total = int(rng.choice([1, 8, 16])), 100
        cu = rng.integers(-2, total + 2, n + 1)
        if rng.random() < 0.5:
            cu[0::2], cu[1::2] = 0, total
        got = _run(program, group, 1, total, 40000, total, cu, rng.integers(0, 40000, n))
        assert got["used"] <= got["room"]
        if got["items"] > got["planned"]:   # only where the first queries are reported
            assert got["status"] == DOMAIN
            over += 1
    assert over


@pytest.mark.parametrize("n,kv_heads,max_q,longest", [(1, 1024, 1 << 14, 1 << 30), (40, 1024, 1 << 14, 1 << 30),
                                                      (4096, 600, 27962, 1 << 29), (3, 1, 1 << 20, 1 << 30)])
def test_steps_beyond_32_bits(program, n, kv_heads, max_q, longest):
    """Steps times row blocks over the target pass 31 bits: the parts are still as planned."""
    got = _run(program, 16 * kv_heads if kv_heads == 1 else kv_heads, kv_heads, max_q, longest, n * max_q,
               np.arange(n + 1) * max_q, [longest] * n)
    assert got["status"] == 0 and got["left"] == 0
    assert got["items"] <= got["planned"]
    assert 0 < got["per"] <= longest // 32
