"""The example runs the operators together: contexts written, requantised, taken to the
host and back, and attended to by trees of drafted tokens."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("agents,tokens,drafts", [(3, 200, 1), (2, 1500, 64)])
def test_resume_agents(agents, tokens, drafts):
    from examples import resume_agents
    found = resume_agents.main(agents, tokens, drafts, seed=1, log=lambda *_: None)
    # 16 bits round-trip exactly; e4m3 rounds a value by at most 2^-4 of itself and e2m1 by at
    # most a quarter (above its smallest step), as relative errors of random sign in the
    # values and of a factor |q||k| / sqrt(dim) ~ 1 to a few in the scores: the two together
    # stay below 1/8 and 1/2 of the output
    assert found["bf16"]["error"] == 0 and found["bf16"]["lse_error"] == 0
    assert 0 < found["fp8"]["error"] < 1 / 8 and 0 < found["fp4"]["error"] < 1 / 2
    assert found["fp8"]["error"] < found["fp4"]["error"]
    assert found["bf16"]["bytes_per_token"] == 131072
    assert found["fp4"]["contexts"] > 3.7 * found["bf16"]["contexts"]
    for kind in found.values():   # restoring costs as the bytes do
        assert kind["b2_per_token"] * 131072 == pytest.approx(
            found["bf16"]["b2_per_token"] * kind["bytes_per_token"], rel=1e-12)
