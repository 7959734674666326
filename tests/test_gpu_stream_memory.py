"""The cost model's wrappers on another stream than torch's current one, with memory that
was freed while the current stream still had to read and write it."""
import pytest

import workloads
from tests.test_gpu_kv_streams import Pending
from tests.test_gpu_streams import LC, _dev, case, kvr  # noqa: F401

pytestmark = pytest.mark.gpu


def _bytes(*tensors):
    return [t.numel() * t.element_size() for t in tensors]


def test_select(kvr):  # noqa: F811
    import torch
    cost = torch.rand((1 << 19, 5, 1, 2), dtype=torch.float64, device="cuda")
    want = kvr.kvr_select_policy(cost, True)
    p = Pending(_bytes(*want))
    got = kvr.kvr_select_policy(cost, True, stream=p.side)
    p.check(*zip(got, want))


@pytest.mark.parametrize("method", ["brute", "sorted"])
def test_cost_grid(kvr, case, method):  # noqa: F811
    import torch
    m = kvr.KVR_BRUTE if method == "brute" else kvr.KVR_SORTED
    n = 1 << 20
    w, T = case["w"].repeat(n // 3001 + 1)[:n], case["T"].repeat(n // 3001 + 1)[:n]
    first = kvr.CostGridCall(w, T, case["prices"], case["grid"], method=m)
    first.launch()
    want, ws = first.cost.clone(), _bytes(first.ws)
    del first
    p = Pending(ws)
    call = kvr.CostGridCall(w, T, case["prices"], case["grid"], method=m)
    call.launch(p.side)
    p.check()
    assert p.took(call.ws) and torch.equal(call.cost, want)
    del call
    p = Pending(ws)
    got = kvr.kvr_cost_grid(w, T, case["prices"], case["grid"], m, stream=p.side, check=False)
    p.check()
    assert torch.equal(got, want)


@pytest.mark.parametrize("factored", [False, True])
def test_bootstrap(kvr, case, factored):  # noqa: F811
    import torch
    args = (case["w"], case["T"], case["idx"], case["prices"], case["grid"])
    first = kvr.BootstrapCall(*args, want_cost=True, factored=factored)
    first.launch()
    want, sizes = [first.best.clone(), first.cost.clone()], _bytes(first.ws, first.cost)
    del first
    p = Pending(sizes)
    got = kvr.kvr_bootstrap(*args, want_cost=True, factored=factored, stream=p.side, check=False)
    p.check()
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[1])


def test_replay_controller_and_crossover(kvr, case):  # noqa: F811
    import torch
    rc = workloads.replay_case("mixture", 3 * LC * 40.0 / 425.0, reps=3, n=2000, seed=77)
    price = kvr.kvr_prices_from_platform(1.0, 1.0, 1.0, 1.0, 1.0, 40.0, 1800.0)
    price.b2_per_token, price.b3_per_token = 0.02, 1.91
    arr, w = _dev(rc.arrival_s, torch.float64), _dev(rc.wait_s, torch.float64)
    lam = 3 * LC * 40.0 / 425.0
    sizes = _bytes(kvr.ControllerCall(arr, w, price, lam).ws)
    replay = kvr.kvr_capacity_replay(arr, w, price, [30.0, 600.0])
    out = bytes(kvr.kvr_controller_select(arr, w, price, lam))
    share = kvr.kvr_crossover_statistic(case["w"], case["prices"])
    p = Pending(sizes)
    got = kvr.kvr_capacity_replay(arr, w, price, [30.0, 600.0], stream=p.side, check=False)
    p.check()
    assert all(torch.equal(x, y) for x, y in zip(got, replay))
    p = Pending(sizes)
    call = kvr.ControllerCall(arr, w, price, lam)
    call.launch(p.side)
    p.check()
    assert bytes(call.result()) == out
    p = Pending(sizes)
    got = kvr.kvr_crossover_statistic(case["w"], case["prices"], stream=p.side, check=False)
    p.check()
    assert all(torch.equal(x, y) for x, y in zip(got, share))
