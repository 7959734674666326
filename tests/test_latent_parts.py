"""How latent attention's sequences are cut into parts, on the host: all parts have a block and room
in the workspace, no CU is left with much more than its share, and no long sequence stays whole
because many short ones are beside it."""
import os
import subprocess

import numpy as np
import pytest

import paper_2608_30830_amd as kvr
from paper_2608_30830_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    if not os.path.exists(kvr.LIB_PATH):
        build.build()
    lib = os.path.dirname(build.LIB)
    exe = str(tmp_path_factory.mktemp("parts") / "latent_parts")
    subprocess.run([build.HIPCC, "--cuda-host-only", "-x", "hip", "-std=c++17", "-O1", "-I" + build.CSRC,
                    "-I" + os.path.join(build.ROOT, "include"), os.path.join(HERE, "latent_parts.cpp"),
                    "-x", "none", build.LIB, "-Wl,-rpath," + lib, "-o", exe], check=True, capture_output=True,
                   timeout=120)

    def call(heads, rank, nq, kv, max_kv=None):
        text = " ".join(str(int(x)) for x in [heads, rank, max(nq), max_kv or max(kv), len(kv), *nq, *kv])
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=60)
        names = ("direct", "planned", "room", "per", "items", "total", "blocks", "longest", "fit", "counts")
        got = dict(zip(names, map(int, out.stdout.split())))
        if not got["direct"]:
            assert got["items"] <= got["planned"]
            assert got["room"] == got["planned"] or got["room"] == 0 and got["per"] >= got["longest"]
        assert got["counts"] <= 12
        return got

    return call


def test_lengths_that_fit(run):
    rng = np.random.default_rng(2)
    for _ in range(150):
        n = int(np.exp(rng.uniform(0, np.log(4096))))
        heads, rank = int(rng.choice([1, 5, 16, 20, 40, 128])), int(rng.choice([256, 512]))
        max_q = int(np.exp(rng.uniform(0, np.log(200))))
        nq = rng.integers(0, max_q + 1, n)
        nq[rng.integers(n)] = max_q
        kv = nq + np.exp(rng.uniform(0, np.log(100000), n)).astype(int)
        got = run(heads, rank, nq, kv)
        if got["blocks"] * 2 <= got["fit"] and not got["direct"]:
            # one round, of parts at most what total / (fit - blocks) gives, or the fewest steps
            assert got["items"] <= got["fit"]
            assert got["per"] <= max(8, got["total"] // (got["fit"] - got["blocks"]) + 1)


@pytest.mark.parametrize("n", [1, 60, 129, 200, 255, 256, 257, 299, 1000, 4000])
def test_one_long_sequence_among_short_ones(run, n):
    got = run(16, 512, [1] * (n + 1), [20] * n + [131072])
    assert got["longest"] == 4096
    assert got["per"] <= 80   # 4,096 steps in 51 or more parts


@pytest.mark.parametrize("n", [64, 130, 200, 256, 300, 400, 512, 700, 2000])
def test_equal_sequences(run, n):
    """Rounds of parts take at most a third more than an even share, and what each part costs."""
    got = run(16, 512, [1] * n, [8192] * n)
    rounds = -(-got["items"] // got["fit"])
    size = -(-got["longest"] // -(-got["longest"] // got["per"]))
    share = got["total"] / got["fit"]
    if n <= 200 or n == 400 or n == 700:
        assert rounds * size <= 1.5 * share + 8 * rounds
    else:
        assert rounds * size <= 2 * share


@pytest.mark.parametrize("bound", [131072, 1 << 30])
def test_a_loose_bound_on_the_lengths(run, bound):
    tight, loose = (run(16, 512, [1] * 40, [4096] * 40, max_kv=m) for m in (None, bound))
    assert tight["per"] == loose["per"] and tight["items"] == loose["items"]


def test_no_tokens(run):
    assert run(16, 512, [1] + [0] * 9, [1] + [0] * 9)["blocks"] == 1
    assert run(128, 256, [3], [3])["items"] >= 1
