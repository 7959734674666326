"""The ways to long contexts by what they promise of each frequency, read off the table, not by
the steps that compute them: which pairs turn often enough to keep theirs, which are
divided by the factor, and what is between."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvr():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_30830_amd as k
    k.load_library()
    return k


def _frequencies(kvr, rot, **kw):
    """w of every pair, from the cosine and sine of position 1 (w <= 1)."""
    row = kvr.kvr_rotary_table(rot, 2, **kw)[1].double().cpu().numpy()
    return np.arctan2(row[1], row[0])


NEAR = dict(rtol=2.0 ** -21, atol=0)   # the cosine's and the sine's rounding to 32 bits


@pytest.mark.parametrize("rot", [2, 64, 100, 256])
@pytest.mark.parametrize("theta", [10000.0, 500000.0])
def test_plain_and_linear(kvr, rot, theta):
    w = _frequencies(kvr, rot, theta=theta)
    assert w[0] == pytest.approx(1.0, rel=2.0 ** -21)
    ratio = w[1:] / w[:-1]                                       # geometric: one ratio, theta^(-2 / rot)
    assert np.allclose(ratio, theta ** (-2.0 / rot), rtol=2.0 ** -20)
    assert np.allclose(_frequencies(kvr, rot, theta=theta, kind=kvr.KVR_ROPE_LINEAR, factor=5.0), w / 5, **NEAR)


@pytest.mark.parametrize("rot", [4, 64, 128])
@pytest.mark.parametrize("factor", [1.0, 3.0, 16.0])
def test_base(kvr, rot, factor):
    """The first pair keeps its frequency and the last one's is divided by the factor."""
    w = _frequencies(kvr, rot, theta=10000.0)
    x = _frequencies(kvr, rot, theta=10000.0, kind=kvr.KVR_ROPE_BASE, factor=factor)
    assert x[0] == pytest.approx(w[0], rel=2.0 ** -20) and x[-1] == pytest.approx(w[-1] / factor, rel=2.0 ** -20)


@pytest.mark.parametrize("rot,theta,trained,low,high", [(128, 500000.0, 8192.0, 1.0, 4.0), (64, 10000.0, 4096.0, 1.0, 32.0),
                                                        (96, 10000.0, 2048.0, 0.5, 3.0), (64, 10000.0, 64.0, 20.0, 30.0)])
def test_blends(kvr, rot, theta, trained, low, high):
    factor = 8.0
    w = theta ** (-2.0 * np.arange(rot // 2) / rot)
    turns = trained * w / (2 * math.pi)
    kw = dict(theta=theta, factor=factor, low=low, high=high, trained_len=trained)
    x = _frequencies(kvr, rot, kind=kvr.KVR_ROPE_TURNS, **kw)
    assert np.allclose(x[turns >= high], w[turns >= high], **NEAR)
    assert np.allclose(x[turns <= low], w[turns <= low] / factor, **NEAR)
    mid = (turns > low) & (turns < high)
    keep = (x / w - 1 / factor) / (1 - 1 / factor)               # share of the unchanged frequency
    assert np.allclose(keep[mid], (turns[mid] - low) / (high - low), rtol=0, atol=2.0 ** -18)
    # by the index: from the last pair with `high` turns or more (or the first) evenly down to the first pair with
    # `low` turns or fewer, among all whole indexes up to rot - 1
    i = np.arange(rot)
    t = trained * theta ** (-2.0 * i / rot) / (2 * math.pi)
    a = i[t >= high].max() if (t >= high).any() else 0
    b = i[t <= low].min() if (t <= low).any() else rot - 1
    x = _frequencies(kvr, rot, kind=kvr.KVR_ROPE_INDEX, **kw)
    j = np.arange(rot // 2)
    assert np.allclose(x[j <= a], w[j <= a], **NEAR)
    assert np.allclose(x[j >= max(b, a + 1)], w[j >= max(b, a + 1)] / factor, **NEAR)
    keep = (x / w - 1 / factor) / (1 - 1 / factor)
    mid = (j > a) & (j < b)
    assert np.allclose(keep[mid], (b - j[mid]) / max(b - a, 1), rtol=0, atol=2.0 ** -18)


def test_magnitude(kvr):
    one, two = (kvr.kvr_rotary_table(64, 50, magnitude=m) for m in (1.0, 2.0))
    import torch
    assert torch.equal(2 * one, two)
