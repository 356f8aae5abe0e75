"""The next-token example: log probabilities, list steps and list synchronizations together in a training run."""
import pytest

from paper_2310_14423_b200 import binding as B
from paper_2310_14423_b200 import next_token
from paper_2310_14423_b200 import workloads as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("states,state_sync", [("f32", "keep"), ("e4m3", "keep"), ("e4m3", "average"), ("e4m3", "reset")])
def test_the_model_learns(states, state_sync):
    r = next_token.train(workers=3, steps=120, vocab=101, width=64, states=states, state_sync=state_sync)
    # most of the way from the first loss to the least possible one
    assert r["start"] > 0.97 * r["uniform"]
    assert r["loss"] < r["entropy_rate"] + 0.35 * (r["start"] - r["entropy_rate"])
    assert r["replicas_equal"]
    w = W.Workload("next_token", 3, W.flat_layout(1), W.OPT_ADAMW, T=120, T_warmup=6, eta_max=8e-3, alpha=0.0175, H_base=4, weight_decay=0.05)
    starts, _ = B.qsr_config_schedule(B.make_config(w))
    assert r["rounds"] == len(starts)
    assert r["launches"] == 2 * 120 + r["rounds"] * (2 if state_sync == "reset" else 1)
