"""The network of examples/mlp_from_svd.py: its gradients against the same network in 64 bits, and a few steps of training.

Tolerances.  An 8-bit code is off by at most half a step of 1/127 of the largest number of its row, about 0.03 standard deviations of a row of a few
hundred normal numbers: an error of 1 % a number, for the inputs, the rest of the weights and the kept inputs alike.  Products over
independent errors keep that: 1.5 % of an output.  The difference to the target is about half an output here, so gradients carry 3 % from it, 1 % from the
kept inputs and as much from the second layer's codes; hidden numbers near zero that change sides add a few more.  0.15 of the norm.
"""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "mlp_from_svd.py")
spec = importlib.util.spec_from_file_location("mlp_from_svd", PATH)
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


def grads64(net, X, target):
    """Mean squared error and its gradients in 64 bits on the CPU, with the weights that the trainer holds."""
    p = [t.detach().double().cpu().requires_grad_() for t in (net.first.W, net.first.bias, net.second.W, net.second.bias)]
    Y = torch.relu(X.double().cpu() @ p[0].t() + p[1]) @ p[2].t() + p[3]
    loss = ((Y - target.double().cpu()) ** 2).mean()
    loss.backward()
    return float(loss.detach()), [t.grad for t in p]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("features,hidden,tokens,rank", [(256, 512, 200, 32), (200, 600, 130, 24)])
def test_gradients(dtype, features, hidden, tokens, rank):
    ctx = example.Rsvd(0)
    W1, b1, W2, b2 = example.network(features, hidden, 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    X = torch.randn(tokens, features, generator=g, device="cuda").to(example.TYPES[dtype])
    target = torch.randn(tokens, features, generator=g, device="cuda")
    net = example.Mlp(ctx, W1, b1, W2, b2, rank)
    loss, want = grads64(net, X, target)
    got = net.step(X, target, 0.0)
    assert abs(got - loss) <= 0.05 * loss
    for name, have, ref in zip(("dW1", "db1", "dW2", "db2"), (net.first.dW, net.first.db, net.second.dW, net.second.db), want):
        error = float((have.double().cpu() * 2 / target.numel() - ref).norm() / ref.norm())
        assert error <= 0.15, (name, error)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_training_lowers_the_error_and_one_token_is_answered(dtype):
    errors, net, Y, one = example.train(256, 512, 300, 32, 5, example.TYPES[dtype])
    assert all(e == e for e in errors) and errors[-1] < errors[0]
    # a token alone: the same codes and integers, the low-rank sums in another order, one rounding of the hidden numbers apart
    scale = float(Y[:1].float().abs().max())
    assert float((one - Y[:1]).float().abs().max()) <= 0.03 * scale
