"""The routed layer's calls inside a torch.autograd.Function, and their refusal outside of one."""
import pytest
import torch

import paper_2403_17017_amd as S
from tests.gpu_util import announce

pytestmark = pytest.mark.gpu


class ThereAndBack(torch.autograd.Function):
    """y = combine(gather(x), weight): each token's row times the sum of its weights."""

    @staticmethod
    def forward(ctx, x, weight, expert):
        r = S.seer_route(expert, 3)
        rows = S.seer_route_gather(r, x)
        ctx.save_for_backward(rows, weight)
        ctx.r = r
        return S.seer_route_combine(r, rows, weight=weight)

    @staticmethod
    def backward(ctx, dy):
        rows, weight = ctx.saved_tensors
        dz, dweight = S.seer_route_grad(ctx.r, dy, rows, weight=weight)
        return S.seer_route_combine(ctx.r, dz), dweight, None


def test_in_a_function_of_autograd():
    announce("routed layer under autograd")
    g = torch.Generator(device="cuda:0").manual_seed(1)
    x = torch.randn(50, 24, generator=g, device="cuda:0", requires_grad=True)
    w = torch.rand(50, 2, generator=g, device="cuda:0", requires_grad=True)
    e = torch.randint(0, 3, (50, 2), generator=g, device="cuda:0")
    c = torch.randn(50, 24, generator=g, device="cuda:0")
    (ThereAndBack.apply(x, w, e) * c).sum().backward()
    near = lambda a, b: bool(((a - b).abs() <= 1e-5 * (1 + b.abs())).all())
    assert near(x.grad, c * w.detach().sum(1, keepdim=True))
    assert near(w.grad, (c * x.detach()).sum(1, keepdim=True).expand(-1, 2))
    r = S.seer_route(e, 3)
    for call in (lambda: S.seer_route_gather(r, x), lambda: S.seer_route_gather(r, x.detach(), weight=w), lambda: S.seer_i8_quantize(x),
                 lambda: S.seer_route_gather_i8(r, x), lambda: S.seer_route_combine(r, torch.cat([x, x]), weight=None)):
        with pytest.raises(RuntimeError, match="history"):
            call()
    with torch.no_grad():
        assert S.seer_route_gather(r, x).shape == (100, 24)
