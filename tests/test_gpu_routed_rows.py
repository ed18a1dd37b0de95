"""seer_route, seer_route_gather, seer_route_combine, seer_route_grad against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2403_17017_amd as S
from oracle import routed_oracle as O
from tests.gpu_util import announce
from tests.routed_util import ROUND, TINY, TYPES, U32, assert_within, choices, host, rounded, shifted, spread

pytestmark = pytest.mark.gpu

SIZES = [  # tokens, choices, experts, skew, padding
    (0, 2, 4, 0, 0), (1, 1, 1, 0, 0), (1, 8, 128, 1, 0), (3, 2, 5, 0, 0.5), (63, 1, 7, 0, 0), (64, 1, 1, 0, 0), (65, 3, 300, 1, 0.1),
    (511, 4, 64, 1, 0.02), (1024, 4, 16, 0, 0), (1025, 4, 1500, 0.5, 0), (700, 6, 4096, 0, 0.1), (5000, 2, 3, 2, 0), (9001, 8, 257, 1, 0.03),
    (70001, 8, 64, 0.5, 0.01),
]


@pytest.mark.parametrize("index", ["int32", "int64"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sort(size, index):
    T, C, E, skew, padding = size
    announce(f"route {size} {index}")
    rng = np.random.default_rng(T + 7 * E)
    e = choices(rng, T, C, E, skew, padding).astype(index)
    if T > 2:
        e[T // 2, 0], e[T - 1, C - 1], e[T // 3, C - 1] = E, -7, np.iinfo(e.dtype).max     # no expert's, either
    r = S.seer_route(torch.from_numpy(e).cuda(), E)
    ptr, order, slots = O.route(e, E)
    assert np.array_equal(host(r.expert_ptr), ptr)
    assert np.array_equal(host(r.slot_choice), order)
    assert np.array_equal(host(r.choice_slot), slots)


def test_nobody_chooses_an_expert():
    e = torch.full((300, 2), -1, dtype=torch.int64, device="cuda:0")
    r = S.seer_route(e, 9)
    assert host(r.expert_ptr).tolist() == [0] * 10 and np.array_equal(host(r.slot_choice), np.arange(600))
    assert np.array_equal(host(r.choice_slot).reshape(-1), -1 - np.arange(600))
    x = torch.randn(300, 40, device="cuda:0")
    assert not S.seer_route_gather(r, x).any()
    z = torch.full((600, 40), float("nan"), device="cuda:0")
    assert not S.seer_route_combine(r, z, weight=torch.ones(300, 2, device="cuda:0")).any()
    dz, dw = S.seer_route_grad(r, x, z)
    assert not dz.any() and not dw.any()


ROWS = [  # tokens, choices, experts, padding, columns
    (1, 8, 128, 0, 2048), (1, 1, 1, 0, 1), (0, 3, 4, 0, 16), (5, 2, 3, 0.4, 0), (7, 3, 4, 0.3, 7), (33, 2, 8, 0, 63), (48, 8, 64, 0, 512),
    (129, 4, 16, 0.05, 1023), (20, 1, 2, 0, 1025), (17, 5, 9, 0.2, 4096), (3, 9, 20, 0, 9001), (2, 17, 40, 0.5, 130), (300, 2, 8, 0.1, 8),
    (4099, 2, 8, 0.1, 33), (4096, 3, 16, 0, 128), (5, 3, 8, 0.2, 260), (4101, 1, 4, 0.3, 100),
]


def case(size, kind, seed):
    T, C, E, padding, D = size
    rng = np.random.default_rng(seed + T + 31 * D)
    e = choices(rng, T, C, E, 0.7, padding)
    r = S.seer_route(torch.from_numpy(e).cuda(), E)
    draw = lambda n: rounded(rng.standard_normal((n, D)) * 10.0 ** rng.integers(-2, 3, (n, 1)), kind)
    w = torch.from_numpy(rng.random((T, C), dtype=np.float32)).cuda()
    return r, O.route(e, E)[2], draw, w


def poison(rows, cols, kind):
    return torch.full((rows, cols), float("nan"), dtype=TYPES[kind], device="cuda:0")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("size", ROWS, ids=str)
def test_rows_to_the_experts_and_back(size, kind):
    announce(f"rows {size} {kind}")
    T, C, _, _, D = size
    r, slots, draw, w = case(size, kind, 1)
    x, z = draw(T), draw(T * C)
    out = S.seer_route_gather(r, x, out=poison(T * C, D, kind))
    assert np.array_equal(host(out), O.gather(slots, host(x)))          # copies
    want = O.gather(slots, host(x), host(w))
    # one product in fp32, one rounding to the type
    assert_within(host(S.seer_route_gather(r, x, weight=w)), want, np.abs(want) * (U32 + ROUND[kind] * (1 + U32)) + TINY[kind], "gather")
    for weight in (None, w):
        want, size_ = O.combine(slots, host(z), None if weight is None else host(w))
        got = host(S.seer_route_combine(r, z, weight=weight, y=poison(T, D, kind)))
        # C products and C sums in fp32, then one rounding
        off = 2 * C * U32 * size_
        assert_within(got, want, off + (np.abs(want) + off) * ROUND[kind] + TINY[kind], "combine")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("size", ROWS, ids=str)
def test_gradients(size, kind):
    announce(f"grad {size} {kind}")
    T, C, _, _, D = size
    r, slots, draw, w = case(size, kind, 2)
    dy, z = draw(T), draw(T * C)
    poisoned = z.clone()
    poisoned[int(host(r.expert_ptr)[-1]):] = float("nan")                     # rows that are no expert's are not read
    for weight in (None, w):
        dz, dw = S.seer_route_grad(r, dy, poisoned, weight=weight, dz=poison(T * C, D, kind))
        want_z, want_w, size_ = O.combine_grad(slots, host(dy), host(z), None if weight is None else host(w))
        assert_within(host(dz), want_z, np.abs(want_z) * (U32 + ROUND[kind] * (1 + U32)) + TINY[kind], "dz")
        assert_within(host(dw), want_w, (D + 1) * U32 * size_ + 2.0 ** -140, "dweight")
    only_w = S.seer_route_grad(r, dy, z, need_dz=False)
    only_z = S.seer_route_grad(r, dy, None, weight=w, need_dweight=False)
    assert only_w[0] is None and only_z[1] is None
    assert torch.equal(only_w[1], S.seer_route_grad(r, dy, z)[1]) and torch.equal(only_z[0], dz)


def test_gradients_against_differences():
    """The sum of c * y moves by the gradients' products with a small step, both ways of the layer."""
    T, C, E, D = 12, 3, 5, 33
    rng = np.random.default_rng(5)
    e = choices(rng, T, C, E, 0.5, 0.2)
    slots = O.route(e, E)[2]
    r = S.seer_route(torch.from_numpy(e).cuda(), E)
    f32 = lambda *s: rng.standard_normal(s).astype(np.float32)
    z, w, c, dz_, dw_ = f32(T * C, D), f32(T, C), f32(T, D), f32(T * C, D), f32(T, C)
    cuda = lambda a: torch.from_numpy(a).cuda()
    gz, gw = S.seer_route_grad(r, cuda(c), cuda(z), weight=cuda(w))
    f = lambda s: np.sum(c.astype(np.float64) * O.combine(slots, z + s * dz_.astype(np.float64), w + s * dw_.astype(np.float64))[0])
    h = 2.0 ** -10
    slope = (f(h) - f(-h)) / (2 * h)                 # exact: f is quadratic in the step
    have = np.sum(host(gz) * dz_) + np.sum(host(gw) * dw_)
    scale = np.sum(np.abs(host(gz) * dz_)) + np.sum(np.abs(host(gw) * dw_))
    assert abs(slope - have) <= (D + 4) * U32 * scale + 1e-9 * scale
    # the way there: out = w * x; its gradients are combine(dout, w) and <x, dout>
    x, dout, dx_ = f32(T, D), f32(T * C, D), f32(T, D)
    gx = S.seer_route_combine(r, cuda(dout), weight=cuda(w))
    gw = S.seer_route_grad(r, cuda(x), cuda(dout), need_dz=False)[1]
    f = lambda s: np.sum(dout.astype(np.float64) * O.gather(slots, x + s * dx_.astype(np.float64), w + s * dw_.astype(np.float64)))
    slope = (f(h) - f(-h)) / (2 * h)
    have = np.sum(host(gx) * dx_) + np.sum(host(gw) * dw_)
    scale = np.sum(np.abs(host(gx) * dx_)) + np.sum(np.abs(host(gw) * dw_))
    assert abs(slope - have) <= (D + 2 * C + 4) * U32 * scale + 1e-9 * scale


@pytest.mark.parametrize("kind", list(TYPES))
def test_rows_apart_and_off_alignment(kind):
    T, C, E, D = 37, 3, 6, 203
    r, slots, draw, w = case((T, C, E, 0.1, D), kind, 3)
    x, z = draw(T), draw(T * C)
    for ld, by in ((D + 5, 1), (256, 0), (D, 3)):
        announce(f"strides {kind} {ld} {by}")
        xs, zs = spread(x, ld), spread(z, ld)
        if ld == D:
            xs, zs = shifted(x, by), shifted(z, by)
        out = spread(poison(T * C, D, kind), ld, 7.0)
        y = spread(poison(T, D, kind), ld, 7.0)
        dz = spread(poison(T * C, D, kind), ld, 7.0)
        assert torch.equal(S.seer_route_gather(r, xs, weight=w, out=out), S.seer_route_gather(r, x, weight=w))
        assert torch.equal(S.seer_route_combine(r, zs, weight=w, y=y), S.seer_route_combine(r, z, weight=w))
        got, want = S.seer_route_grad(r, xs, zs, weight=w, dz=dz), S.seer_route_grad(r, x, z, weight=w)
        assert torch.equal(got[0], want[0])
        tol = (D + 1) * U32 * O.combine_grad(slots, host(x), host(z))[2] * 2
        assert_within(host(got[1]), host(want[1]), tol, "dweight")
        if ld > D:                                      # nothing between the rows is written
            for t in (out, y, dz):
                between = t.as_strided((t.shape[0] - 1, ld - D), (ld, 1), t.storage_offset() + D)
                assert bool((between == 7.0).all())


def test_infinities_and_nan_stay_where_they_are():
    e = torch.tensor([[0, 1], [1, -1], [-1, -1], [0, 1]], device="cuda:0")
    r = S.seer_route(e, 2)
    z = torch.ones(8, 16, device="cuda:0")
    slots = r.choice_slot.cpu()
    z[int(slots[0, 1]), 3] = float("inf")
    z[int(slots[3, 0]), 5] = float("nan")
    z[int(r.expert_ptr[-1]):] = float("nan")
    w = torch.tensor([[1.0, 2.0], [1.0, float("inf")], [float("nan"), 1.0], [1.0, 1.0]], device="cuda:0")
    y = host(S.seer_route_combine(r, z, weight=w))
    assert y[0, 3] == np.inf and np.isnan(y[3, 5])
    y[0, 3] = y[3, 5] = 0
    assert np.isfinite(y).all() and (y[1] == 1).all() and (y[2] == 0).all()


def test_captured_and_on_another_stream():
    T, C, E, D = 500, 4, 16, 256
    rng = np.random.default_rng(9)
    e = torch.from_numpy(choices(rng, T, C, E, 1, 0.05)).cuda()
    x = torch.randn(T, D, device="cuda:0").bfloat16()
    w = torch.rand(T, C, device="cuda:0")

    def step(stream=None):
        r = S.seer_route(e, E, stream=stream)
        rows = S.seer_route_gather(r, x, stream=stream)
        y = S.seer_route_combine(r, rows, weight=w, stream=stream)
        dz, dw = S.seer_route_grad(r, x, rows, weight=w, stream=stream)
        return r.choice_slot, rows, y, dz, dw
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_refusals():
    e = torch.zeros(4, 2, dtype=torch.int64, device="cuda:0")
    r = S.seer_route(e, 3)
    x = torch.zeros(4, 8, device="cuda:0")
    with pytest.raises(ValueError):
        S.seer_route(e.cpu(), 3)
    with pytest.raises(ValueError):
        S.seer_route(e.float(), 3)
    with pytest.raises(S.SeerError):
        S.seer_route(e, 0)
    with pytest.raises(S.SeerError):
        S.seer_route(e, 4097)
    with pytest.raises(ValueError):
        S.seer_route_gather(r, x.t())
    with pytest.raises(TypeError):
        S.seer_route_gather(r, x.double(), out=x)
    with pytest.raises(S.SeerError):
        S.seer_route_gather(r, x[:3])
    with pytest.raises(S.SeerError):
        S.seer_route_gather(r, x, out=torch.zeros(8, 8, device="cuda:0").bfloat16())
    with pytest.raises(ValueError):
        S.seer_route_gather(r, x, weight=torch.zeros(4, 2, device="cuda:0").bfloat16())
    with pytest.raises(S.SeerError):
        S.seer_route_combine(r, x)
    z = torch.zeros(8, 8, device="cuda:0")
    with pytest.raises(S.SeerError):
        S.seer_route_combine(r, z, y=z[:4])              # y lies in z
    with pytest.raises(S.SeerError):
        S.seer_route_grad(r, x, None)                    # dweight needs z
    with pytest.raises(S.SeerError):
        S.seer_route_gather(r, x[:1].expand(4, 8))       # rows on top of one another
    with pytest.raises(ValueError):
        S.seer_route_gather(r, x, stream=torch.cuda.current_stream().cuda_stream)
