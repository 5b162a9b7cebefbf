"""The training program of examples/train_policy.py learns: embedding, gate network, MoE layer, policy loss and both
optimizers together."""
import pytest

pytestmark = pytest.mark.gpu


def test_rewards_rise():
    from examples.train_policy import train
    rewards = train(iterations=40)
    assert rewards[0] < 0.1                      # 61 answers: one in 61 is right by chance
    assert sum(rewards[-5:]) / 5 > 0.6
