"""The example of a routed layer: its gradients, training, and serving in 8-bit integers."""
import pytest
import torch

from paper_2403_17017_amd.routed_layer import RoutedLayer, main

pytestmark = pytest.mark.gpu


def test_gradients_of_the_whole_layer():
    """Against automatic differentiation of the formula in 64 bits, with the same experts chosen."""
    layer = RoutedLayer(experts=4, choices=2, columns=20, hidden=24, seed=4)
    g = torch.Generator(device="cuda:0").manual_seed(5)
    x, c = (torch.randn(50, 20, generator=g, device="cuda:0") for _ in range(2))
    y, kept = layer.forward(x)
    dx = layer.backward(c, kept)
    leaf = lambda t: t.detach().double().cpu().requires_grad_()
    x64, router, w1, w2 = leaf(x), leaf(layer.router), leaf(layer.w1), leaf(layer.w2)
    expert = kept[2].cpu()
    weight = torch.softmax((x64 @ router.t()).gather(1, expert), dim=1)
    want = 0
    for k in range(2):
        hidden = torch.relu((w1[expert[:, k]] @ x64[:, :, None])[:, :, 0])
        want = want + weight[:, k, None] * (w2[expert[:, k]] @ hidden[:, :, None])[:, :, 0]
    (want * c.double().cpu()).sum().backward()
    # sums of at most some hundred fp32 terms: 2^-24 of their magnitudes each, which are within a factor of ten of the results
    near = lambda got, ref: float((got.double().cpu() - ref).norm()) <= 1e-4 * float(ref.norm())
    assert near(y, want.detach()) and near(dx, x64.grad) and near(layer.grads[0], router.grad)
    for e in range(4):
        assert near(layer.grads[1 + e], w1.grad[e]) and near(layer.grads[5 + e], w2.grad[e])


def test_trained_and_served():
    losses, off = main(["--tokens", "2000", "--steps", "100"])
    assert losses[-1] < 0.6 * losses[0]
    # a 7-bit mantissa for each operand of two products: each value is off by up to 1 / 254 of its row's largest, two operands
    # and two products in quadrature with rows whose largest is some 3 to 4 times the root mean square
    assert off < 0.03
