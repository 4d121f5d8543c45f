"""What a layer and a context keep between calls: a layer's tensors whose values change."""
import pytest
import torch

from gpu_util import ctx
from test_gpu_layer8 import BF16, TYPES, activations, check, gen, grad_reference, product_reference, weight

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [3, 150])
def test_changed_tensors_are_what_the_next_calls_take(dtype, tokens):
    """Both passes against a layer made of the changed tensors, bit for bit, and against the definition with the factors of the forward pass."""
    from paper_2110_03423_amd import Weight8
    g = gen(tokens)
    w = weight(g, 90, 130, 12)
    x, dy = activations(g, tokens, 130, TYPES[dtype]), activations(g, tokens, 90, TYPES[dtype])
    ctx().rsvd_q8_product(x, w), ctx().rsvd_q8_product_grad(dy, w)
    for change in (w.U, w.Vt, w.scale, w.bias):
        change.data.mul_(-0.75)
        change[0] = 0.5
        w.codes.neg_()
        other = Weight8(w.codes.clone(), w.scale.clone(), w.U.clone(), w.Vt.clone(), w.bias.clone())
        y, dx = ctx().rsvd_q8_product(x, w), ctx().rsvd_q8_product_grad(dy, w)
        assert torch.equal(y, ctx().rsvd_q8_product(x, other)) and torch.equal(dx, ctx().rsvd_q8_product_grad(dy, other))
        check(y, *product_reference(x, w), "product")
        want = dy.double() @ (w.codes.double() * w.scale.double()[:, None] + w.U.double() @ w.Vt.double())
        check(dx, want, grad_reference(dy, other)[1], "gradient")


def test_a_captured_gradient_takes_the_factors_of_the_replay():
    g = gen(3)
    w = weight(g, 90, 130, 12)
    dy = activations(g, 100, 90, BF16)
    ctx().rsvd_q8_product_grad(dy, w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dx = ctx().rsvd_q8_product_grad(dy, w)
    for trial in range(4):
        w.U.mul_(-0.5)
        w.Vt[trial] = 1.0
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dx, ctx().rsvd_q8_product_grad(dy, w))
        torch.cuda.synchronize()
