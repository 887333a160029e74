"""The example that runs the codec and the operators around it together: its gradient against
autograd, and that it learns."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_lm_step", os.path.join(ROOT, "examples", "train_lm_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradient_is_autograds():
    """fp32 on both sides over sums of 256 to 1003 terms: 1e-4 of each matrix's gradient."""
    m = example()
    model, data = m.Model(3), m.Bigrams(4)
    tokens, targets = data.batch(256)
    grad = torch.zeros(model.length, device="cuda")
    loss = model.loss_and_gradient(tokens, targets, grad, entropy_reward=0.05)
    ps = [p.clone().requires_grad_() for p in model.views(model.params)]
    emb, up, down, out = ps
    x = emb[tokens]
    logp = torch.log_softmax((x + torch.tanh(x @ up.T) @ down.T) @ out.T, dim=1)
    want = -logp.gather(1, targets[:, None]).mean()
    (want + 0.05 * (logp.exp() * logp).sum(1).mean()).backward()
    assert abs(loss.item() - want.item()) <= 1e-5 * want.item()
    for g, p in zip(model.views(grad), ps):
        assert (g - p.grad).norm() <= 1e-4 * p.grad.norm()


def test_it_learns_through_the_codec():
    m = example()
    losses, floor = m.train(40, 3, batch=1024)
    assert all(math.isfinite(x) for x in losses)
    assert abs(losses[0] - math.log(m.VOCAB)) < 1.0
    assert losses[-1] < 0.6 * losses[0] and losses[-1] > floor - 0.05
