"""The routed layer's calls keep no history for autograd, and say so where torch records one (without a GPU: tensors that are
described only; every call is refused in one way or another)."""
import pytest
import torch

from paper_2403_17017_amd import routed as R
from tests.marshal_util import Described, DescribedRouting

FAR = 1 << 40
T, C, E, D = 4, 2, 3, 8


def mat(rows, cols, at, wanted, dtype=torch.float32):
    return Described((rows, cols), dtype, at * FAR, requires_grad=wanted)


def vec(n, at, wanted):
    return Described((n,), torch.float32, at * FAR, requires_grad=wanted)


CALLS = {   # how many floating tensors, and the call with the i-th of them (or none) requiring grad; its result lies on its input
    "gather": (3, lambda m, r, w: m.gather(r, mat(T, D, 2, w == 0), mat(T * C, D, 2, w == 1), mat(T, C, 3, w == 2), 0)),
    "combine": (3, lambda m, r, w: m.combine(r, mat(T * C, D, 2, w == 0), mat(T, D, 2, w == 1), mat(T, C, 3, w == 2), 0)),
    "grad": (5, lambda m, r, w: m.grad(r, mat(T, D, 2, w == 0), mat(T * C, D, 3, w == 1), mat(T, C, 4, w == 2), mat(T * C, D, 2, w == 3), mat(T, C, 5, w == 4), 0)),
    "quantize": (2, lambda m, r, w: m.quantize(None, mat(T, D, 2, w == 0), mat(T, D, 2, False, torch.int8), vec(T, 3, w == 1), 0)),
    "gather_i8": (2, lambda m, r, w: m.quantize(r, mat(T, D, 2, w == 0), mat(T * C, D, 2, False, torch.int8), vec(T * C, 3, w == 1), 0)),
    "product": (3, lambda m, r, w: m.product(mat(T, D, 2, False, torch.int8), vec(T, 3, w == 0), mat(6, D, 4, False, torch.int8), vec(6, 5, w == 1), None,
                                             mat(T, 6, 2, w == 2), None, 0)),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_tensors_that_require_grad(name):
    m, r = R._ready(), DescribedRouting(T, C, E, FAR)
    tensors, call = CALLS[name]
    assert call(m, r, None) < 0                              # the library's own refusal
    for which in range(tensors):
        with pytest.raises(RuntimeError, match="history"):
            call(m, r, which)
        with torch.no_grad():
            assert call(m, r, which) < 0
    asked = []

    class Function(torch.autograd.Function):                 # what the message says: no history is recorded in a forward
        @staticmethod
        def forward(ctx, x):
            asked.append(call(m, r, 0))
            return x.clone()
    Function.apply(torch.ones(1, requires_grad=True))
    assert asked[0] < 0
