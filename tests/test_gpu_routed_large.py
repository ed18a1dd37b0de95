"""Offsets beyond 32 bits in the routed layer's operators: a few rows are checked in matrices of over 2^31 elements."""
import numpy as np
import pytest
import torch

import paper_2403_17017_amd as S
from tests.gpu_util import announce
from tests.routed_util import U32, host

pytestmark = pytest.mark.gpu


def test_rows():
    announce("routed rows beyond 2^31 elements")
    T, C, E, D = 70000, 8, 16, 4096
    assert T * C * D > 2 ** 31
    g = torch.Generator(device="cuda:0").manual_seed(1)
    e = torch.randint(0, E, (T, C), generator=g, device="cuda:0")
    x = torch.randn(T, D, generator=g, device="cuda:0").bfloat16()
    w = torch.rand(T, C, generator=g, device="cuda:0")
    r = S.seer_route(e, E)
    rows = S.seer_route_gather(r, x)
    some = torch.tensor([0, 1, T // 2, T - 2, T - 1], device="cuda:0")
    slots = r.choice_slot[some].long()
    assert int(slots.max()) * D > 2 ** 31
    assert torch.equal(rows[slots], x[some][:, None, :].expand(-1, C, -1))
    y = S.seer_route_combine(r, rows, weight=w)
    want = x[some].double() * w[some].double().sum(1, keepdim=True)
    # C products and sums in fp32, one rounding to bf16
    assert bool(((y[some].double() - want).abs() <= want.abs() * (2 * C * U32 + 2.0 ** -8)).all())
    dz, dw = S.seer_route_grad(r, x, rows, weight=w)
    want = x[some].double()[:, None, :] * w[some].double()[:, :, None]
    assert bool(((dz[slots].double() - want).abs() <= want.abs() * (U32 + 2.0 ** -8)).all())
    dots = (x[some].double() ** 2).sum(1, keepdim=True).expand(-1, C)
    assert bool(((dw[some].double() - dots).abs() <= dots * (D + 1) * U32).all())
    del rows, dz
    q, s = S.seer_route_gather_i8(r, x)
    qx, sx = S.seer_i8_quantize(x[some])
    assert torch.equal(q[slots], qx[:, None, :].expand(-1, C, -1)) and torch.equal(s[slots], sx[:, None].expand(-1, C))


@pytest.mark.parametrize("rows", [12, 700])
def test_products(rows):
    announce(f"8-bit product with weights beyond 2^32 bytes, {rows} rows")
    G, N, K = 5, 24000, 40000
    assert (G - 1) * N * K < 2 ** 32 < G * N * K
    g = torch.Generator(device="cuda:0").manual_seed(2)
    b = torch.randint(-127, 128, (G, N, K), dtype=torch.int8, device="cuda:0", generator=g)
    a = torch.randint(-127, 128, (rows, K), dtype=torch.int8, device="cuda:0", generator=g)
    sa, sb = torch.rand(rows, generator=g, device="cuda:0"), torch.rand(G, N, generator=g, device="cuda:0")
    ptr = torch.tensor([0, 1, 2, 2, 3, rows], dtype=torch.int32, device="cuda:0")
    y = S.seer_i8_product(a, sa, b, sb, group_ptr=ptr, dtype=torch.float32)
    some = torch.tensor([0, 1, N // 2, N - 1], device="cuda:0")
    for i, e in ((0, 0), (2, 3), (rows - 1, 4), (rows // 2, 4)):
        sums = (b[e, some].cpu().to(torch.int64) * a[i].cpu().to(torch.int64)).sum(1).double()
        want = sums * float(sa[i]) * sb[e, some].double().cpu()
        assert bool(((y[i, some].double().cpu() - want).abs() <= want.abs() * 4.1 * U32).all())


def test_results_beyond_2_31():
    announce("8-bit product with results beyond 2^31 elements")
    M, N, K = 70000, 32000, 64
    g = torch.Generator(device="cuda:0").manual_seed(3)
    a, b = (torch.randint(-127, 128, (n, K), dtype=torch.int8, device="cuda:0", generator=g) for n in (M, N))
    y = S.seer_i8_product(a, torch.ones(M, device="cuda:0"), b, torch.ones(1, N, device="cuda:0"), dtype=torch.float32)
    for i in (0, M // 2, M - 1):
        assert torch.equal(y[i].cpu(), (b.cpu().int() @ a[i].cpu().int()).float())


def test_norm_of_a_tensor_beyond_2_32():
    announce("norm of 2^32 + 12345 elements")
    n = 2 ** 32 + 12345
    t = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda:0")
    t[-1] = 1024
    want = np.sqrt(0.25 * (n - 1) + 1024.0 ** 2)
    assert abs(float(S.seer_grad_norm([t])) - want) <= 1.001 * U32 * want
    norm = S.seer_grad_clip([t], 1.0)
    by = 1.0 / (float(norm) + 1e-6)
    assert abs(float(t[-1]) - 1024 * by) <= 1024 * by * 2.0 ** -7 and abs(float(t[2 ** 32 + 5]) - 0.5 * by) <= 0.5 * by * 2.0 ** -7
    assert bool((t[:-1][:: 2 ** 20] == t[0]).all())
