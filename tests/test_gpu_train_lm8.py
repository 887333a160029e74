"""The example with its hidden layer in 8 bits: its gradient against autograd of the layer without 8 bits, and
that it runs through the codec."""
import math

import pytest
import torch

from test_gpu_train_lm import example

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [256, 77])
def test_gradient_is_near_autograds(n):
    """An operand's rounding to e4m3 is 2^-4 of an entry at most, 2^-4 / sqrt(3) of a norm where errors spread evenly;
    up to four products with two such operands each follow each other on the way to a gradient:
    sqrt(8) / sqrt(3) / 16 = 0.10.  The output matrix is multiplied in 32 bits behind two of them."""
    m = example()
    model, data = m.GatedModel(3), m.Bigrams(4)
    tokens, targets = data.batch(n)
    grad = torch.full((model.length,), float("nan"), device="cuda")
    loss = model.loss_and_gradient(tokens, targets, grad, entropy_reward=0.05)
    ps = [p.double().requires_grad_() for p in model.views(model.params)]
    emb, norm, gate, up, down, out = ps
    x = emb[tokens]
    v = x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-6) * norm
    g = v @ gate.T
    logp = torch.log_softmax((x + (g * torch.sigmoid(g) * (v @ up.T)) @ down.T) @ out.T, dim=1)
    want = -logp.gather(1, targets[:, None]).mean()
    (want + 0.05 * (logp.exp() * logp).sum(1).mean()).backward()
    assert abs(loss.item() - want.item()) <= 0.05 * want.item()
    for got, p in zip(model.views(grad), ps):
        assert (got.double() - p.grad).norm() <= 0.10 * p.grad.norm()


def test_it_runs_through_the_codec():
    m = example()
    losses, _ = m.train(6, 3, batch=512, eight_bit=True)
    assert len(losses) == 6 and all(math.isfinite(x) for x in losses)
    assert abs(losses[0] - math.log(m.VOCAB)) < 1.0
