"""The example that runs the operators together: sampling by the decode step, and policy updates on the sample."""
import importlib.util
import os

import pytest
import torch

from paper_2606_01294_gb300 import ccq

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "policy_step.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("policy_step", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_decode_and_training_forward_agree(example):
    model = example.Model(300, 2, seed=3)
    ids = torch.randint(0, 300, (3, 20), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    with torch.no_grad():
        whole = model.forward(ids).float()
        states = [ccq.CCQState.zeros(3, example.HEADS, example.D, example.D, "cuda") for _ in model.layers]
        one = torch.stack([model.forward(ids[:, t].contiguous(), states).float() for t in range(20)], 1)
    # bf16 activations through two layers: the forward's stated tolerance of 2e-2, once a layer
    assert float((whole - one).abs().max()) <= 2 * 2e-2 * float(whole.abs().max())


def test_policy_updates_raise_the_reward(example):
    rewards = example.train(steps=25, batch=16, length=32, vocab=256, layers=1)
    # 512 tokens a round: a mean reward of one half has a deviation of 0.022, five rounds' mean 0.01
    assert abs(sum(rewards[:2]) / 2 - 0.5) < 0.15
    assert sum(rewards[-5:]) / 5 > sum(rewards[:2]) / 2 + 0.1
