"""seer_i8_quantize, seer_route_gather_i8 and seer_i8_product against their definitions."""
import numpy as np
import pytest
import torch

import paper_2403_17017_amd as S
from oracle import routed_oracle as O
from tests.gpu_util import announce
from tests.routed_util import ROUND, TINY, TYPES, U32, assert_within, choices, host, rounded, shifted, spread

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("shape", [(1, 1), (1, 8192), (3, 15), (5, 16), (4, 17), (33, 1000), (2, 9001), (0, 8), (64, 4096), (3, 0), (9, 1024), (7, 1040), (5, 4112), (3, 8208), (2, 16384), (2, 16400)], ids=str)
def test_quantize(shape, kind):
    announce(f"quantize {shape} {kind}")
    rng = np.random.default_rng(shape[1])
    x = rounded(rng.standard_normal(shape) * 10.0 ** rng.integers(-3, 3, (shape[0], 1)), kind)
    if shape[0] > 2 and shape[1]:
        x[1] = 0
        x[2] = x[2].abs().max() * torch.linspace(-1, 1, shape[1], device="cuda:0")
    q, s = S.seer_i8_quantize(x)
    want_q, want_s = O.quantize(host(x))
    assert np.array_equal(host(s).astype(np.float32), want_s)
    assert np.array_equal(host(q), want_q)
    if q.stride(0) > shape[1] and q.numel():
        room = q.as_strided((shape[0], q.stride(0)), (q.stride(0), 1))
        assert not room[:, shape[1]:].any()              # zeros up to the next multiple of 16
    apart = torch.full((shape[0], shape[1] + 37), 55, dtype=torch.int8, device="cuda:0")
    x2 = spread(x, shape[1] + 3) if shape[1] else x
    q2, _ = S.seer_i8_quantize(x2, q=apart[:, : shape[1]])
    assert torch.equal(q2, q) and bool((apart[:, -(-shape[1] // 16) * 16:] == 55).all())


def test_quantize_at_the_ends_of_the_range():
    x = torch.tensor([[1e-45, 0, 0], [3e38, -3e38, 1e38], [1e-38, -1e-38, 4e-39], [float("inf"), 1, 0], [float("nan"), 1, 2]], device="cuda:0")
    q, s = S.seer_i8_quantize(x)
    want_q, want_s = O.quantize(host(x)[:3])
    assert np.array_equal(host(q)[:3], want_q) and np.array_equal(host(s).astype(np.float32)[:3], want_s)
    assert np.isinf(host(s)[3]) and np.isnan(host(s)[4])
    b = torch.ones(1, 2, 3, dtype=torch.int8, device="cuda:0")
    y = host(S.seer_i8_product(q, s, b, torch.ones(1, 2, device="cuda:0"), dtype=torch.float32))
    assert np.isfinite(y[:3]).all() and not np.isfinite(y[3:]).any()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("size", [(1, 8, 128, 0, 2048), (33, 2, 8, 0.2, 63), (7, 3, 4, 0.3, 7), (129, 4, 16, 0.05, 1030), (2, 17, 40, 0.5, 9001)], ids=str)
def test_quantized_on_the_way_to_the_experts(size, kind):
    announce(f"gather_i8 {size} {kind}")
    T, C, E, padding, D = size
    rng = np.random.default_rng(T)
    r = S.seer_route(torch.from_numpy(choices(rng, T, C, E, 0.7, padding)).cuda(), E)
    x = rounded(rng.standard_normal((T, D)), kind)
    q, s = S.seer_route_gather_i8(r, x)
    qx, sx = S.seer_i8_quantize(x)
    slots = host(r.choice_slot)
    assert np.array_equal(host(q), O.gather(slots, host(qx).astype(np.float64)))
    assert np.array_equal(host(s)[:, None], O.gather(slots, host(sx)[:, None]))


def i8(rng, *shape):
    return torch.from_numpy(rng.integers(-127, 128, shape).astype(np.int8)).cuda()


def check_product(a, b, group_ptr, kind, rng, out=None):
    rows, groups, channels = a.shape[0], b.shape[0], b.shape[1]
    sa = torch.from_numpy((rng.random(rows) * 1e-2 + 1e-3).astype(np.float32)).cuda()
    sb = torch.from_numpy((rng.random((groups, channels)) * 1e-2 + 1e-3).astype(np.float32)).cuda()
    ptr = None if group_ptr is None else torch.tensor(group_ptr, dtype=torch.int32, device="cuda:0")
    if out is None:
        out = torch.full((rows, channels), float("nan"), dtype=TYPES[kind], device="cuda:0")
    S.seer_i8_product(a, sa, b, sb, group_ptr=ptr, out=out)
    want = O.i8_product(host(a), host(sa).astype(np.float32), host(b), host(sb).astype(np.float32), group_ptr)
    # an exact sum, its rounding to fp32, two products there, one rounding to the type
    off = 3.1 * U32 * np.abs(want)
    assert_within(host(out), want, off + (np.abs(want) + off) * ROUND[kind] + TINY[kind], "product")


SHAPES = [  # rows, channels, columns
    (1, 1, 1), (1, 16, 64), (1, 4096, 1024), (3, 5, 7), (16, 16, 128), (17, 33, 100), (64, 64, 256), (65, 129, 272), (128, 256, 4112),
    (200, 300, 96), (257, 511, 1040), (300, 260, 2048), (33, 70, 0), (5, 200, 9000), (512, 512, 512), (1000, 24, 640), (31, 1025, 31),
    (2, 100, 4096), (8, 1000, 2064), (40, 256, 512), (700, 777, 208),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_one_matrix(shape, kind):
    announce(f"i8 {shape} {kind}")
    rng = np.random.default_rng(sum(shape))
    M, N, K = shape
    check_product(i8(rng, M, K), i8(rng, 1, N, K), None, kind, rng)


GROUPS = [  # lengths of the groups, rows behind them, channels, columns
    ([3, 0, 5, 1], 0, 32, 64), ([0, 0, 0], 7, 20, 48), ([64, 128, 0, 65, 1], 3, 130, 272), ([1] * 70, 0, 64, 128), ([0] * 200 + [9] + [0] * 30, 2, 48, 96),
    ([300, 2, 0, 700, 17], 11, 256, 512), ([40, 33, 31, 16, 15, 17, 64, 1], 0, 96, 1024), ([2, 1, 3, 0, 2], 0, 512, 2048), ([500], 12, 64, 160),
    ([5, 260, 255, 256, 257], 0, 300, 144), ([2, 3], 1, 33, 77),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("groups", GROUPS, ids=lambda g: f"{len(g[0])}x{sum(g[0])}+{g[1]}-{g[2]}-{g[3]}")
def test_groups(groups, kind):
    lengths, more, N, K = groups
    announce(f"i8 groups {lengths} {kind}")
    rng = np.random.default_rng(N + K)
    M = sum(lengths) + more
    check_product(i8(rng, M, K), i8(rng, len(lengths), N, K), np.concatenate([[0], np.cumsum(lengths)]).tolist(), kind, rng)


def test_rows_behind_the_groups_are_zero_whatever_they_hold():
    rng = np.random.default_rng(1)
    a, b = i8(rng, 20, 64), i8(rng, 2, 32, 64)
    sa = torch.full((20,), float("nan"), device="cuda:0")
    sa[:9] = 1
    y = S.seer_i8_product(a, sa, b, torch.ones(2, 32, device="cuda:0"), group_ptr=torch.tensor([0, 4, 9], dtype=torch.int32, device="cuda:0"))
    assert not y[9:].any() and bool(torch.isfinite(y.float()).all())


def test_offsets_out_of_range_are_taken_as_the_nearer_end():
    rng = np.random.default_rng(2)
    for M in (20, 700):
        check_product(i8(rng, M, 64), i8(rng, 3, 32, 64), [0, 4, M + 9, M + 10], "f32", rng)


@pytest.mark.parametrize("where", ["apart", "shifted", "odd apart", "out apart"])
@pytest.mark.parametrize("shape", [(5, 70, 256), (150, 270, 512)], ids=str)
def test_strides_and_alignment(shape, where):
    announce(f"i8 {shape} {where}")
    rng = np.random.default_rng(3)
    M, N, K = shape
    a, b = i8(rng, M, K), i8(rng, 1, N, K)
    out = None
    if where == "apart":
        a, b = spread(a, K + 48, 99), spread(b[0], K + 16, 99)[None]
    elif where == "odd apart":
        a, b = spread(a, K + 5, 99), spread(b[0], K + 3, 99)[None]
    elif where == "shifted":
        a, b = shifted(a, 4), shifted(b, 1)
    else:
        out = spread(torch.zeros(M, N, dtype=torch.bfloat16, device="cuda:0"), N + 9, 7.0)
    check_product(a, b, None, "bf16", rng, out)
    if out is not None:
        assert bool((out.as_strided((M - 1, 9), (N + 9, 1), N) == 7.0).all())


def test_the_largest_sums_are_exact():
    K = 131071
    for M, N in ((1, 16), (70, 64), (97, 300)):
        a = torch.full((M, K), -128, dtype=torch.int8, device="cuda:0")
        b = torch.full((1, N, K), -128, dtype=torch.int8, device="cuda:0")
        b[0, 1] = 127
        y = S.seer_i8_product(a, torch.ones(M, device="cuda:0"), b, torch.ones(1, N, device="cuda:0"), dtype=torch.float32)
        want = np.full((M, N), np.float32(K * 16384))
        want[:, 1] = np.float32(-K * 16256)
        assert np.array_equal(host(y), want)


def test_captured():
    rng = np.random.default_rng(4)
    T, C, E, D, N = 40, 2, 8, 512, 384
    e = torch.from_numpy(choices(rng, T, C, E, 1, 0)).cuda()
    x = torch.randn(T, D, device="cuda:0").bfloat16()
    b, sb = i8(rng, E, N, D), torch.rand(E, N, device="cuda:0")

    def step():
        r = S.seer_route(e, E)
        q, s = S.seer_route_gather_i8(r, x)
        return S.seer_i8_product(q, s, b, sb, group_ptr=r.expert_ptr)
    want = step().clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r = S.seer_route(e, E, stream=side)
    q, s = S.seer_route_gather_i8(r, x, stream=side)
    got = S.seer_i8_product(q, s, b, sb, group_ptr=r.expert_ptr, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_refusals():
    a = torch.zeros(4, 64, dtype=torch.int8, device="cuda:0")
    b = torch.zeros(2, 8, 64, dtype=torch.int8, device="cuda:0")
    sa, sb = torch.ones(4, device="cuda:0"), torch.ones(2, 8, device="cuda:0")
    ptr = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda:0")
    S.seer_i8_product(a, sa, b, sb, group_ptr=ptr)
    with pytest.raises(S.SeerError):
        S.seer_i8_product(a, sa, b, sb)                                  # two matrices and no groups
    with pytest.raises(ValueError):
        S.seer_i8_product(a, sa, b, sb, group_ptr=ptr.long())
    with pytest.raises(ValueError):
        S.seer_i8_product(a, sa[:3], b, sb, group_ptr=ptr)
    with pytest.raises(S.SeerError):
        S.seer_i8_product(a[:, :32], sa, b, sb, group_ptr=ptr)
    with pytest.raises(ValueError):
        S.seer_i8_product(a, sa, b.float(), sb, group_ptr=ptr)
    with pytest.raises(TypeError):
        S.seer_i8_product(a, sa, b, sb, group_ptr=ptr, out=torch.zeros(4, 8, device="cuda:0"), dtype=torch.float16)
    with pytest.raises(S.SeerError):
        S.seer_i8_product(a, sa, b, sb, group_ptr=ptr, out=torch.zeros(4, 8, dtype=torch.int8, device="cuda:0"))
    with pytest.raises(S.SeerError) as e:
        S.seer_i8_product(torch.zeros(1, 131072, dtype=torch.int8, device="cuda:0"), sa[:1], torch.zeros(1, 2, 131072, dtype=torch.int8, device="cuda:0"),
                          torch.ones(1, 2, device="cuda:0"))
    assert e.value.status == -6
    with pytest.raises(S.SeerError):
        S.seer_i8_quantize(torch.zeros(4, 8, device="cuda:0"), q=a)


def test_memory_that_ends_before_the_last_rows_zeros_is_refused():
    x = torch.randn(3, 20, device="cuda:0")
    whole = torch.full((2 * 40 + 32,), 55, dtype=torch.int8, device="cuda:0")
    S.seer_i8_quantize(x, q=whole.as_strided((3, 20), (40, 1)))
    assert not whole.as_strided((3, 12), (40, 1), 20).any() and bool((whole.as_strided((2, 8), (40, 1), 32) == 55).all())
    short = torch.zeros(2 * 40 + 31, dtype=torch.int8, device="cuda:0").as_strided((3, 20), (40, 1))
    with pytest.raises(ValueError):
        S.seer_i8_quantize(x, q=short)
    r = S.seer_route(torch.zeros(3, 1, dtype=torch.int64, device="cuda:0"), 1)
    with pytest.raises(ValueError):
        S.seer_route_gather_i8(r, x, q=short)
    S.seer_i8_quantize(x, q=torch.zeros(2 * 25 + 25, dtype=torch.int8, device="cuda:0").as_strided((3, 20), (25, 1)))   # up to ld


@pytest.mark.parametrize("kind", list(TYPES))
def test_quantize_at_and_beside_the_middle(kind):
    """Quotients at n + 1/2 and a few units in the last place to either side: the division decides."""
    base = np.array([127.0, 3.3, 1e-3, 0.7, 2.0 ** -99, 2.0 ** -101, 1.7e38, 1.0 / 3]) if kind != "f16" else np.array([127.0, 3.3, 0.11, 0.7, 60000.0])
    rows = []
    for top in base:
        top = np.float64(np.float32(top))
        scale = np.float32(top) / np.float32(127)
        half = np.arange(-126.5, 127, 1.0).astype(np.float64) * np.float64(scale)
        near = np.concatenate([half * (1 + k * 2.0 ** -23) for k in range(-3, 4)])
        rows.append(np.concatenate([[top], near]))
    x = rounded(np.array(rows), kind)
    q, s = S.seer_i8_quantize(x)
    want_q, want_s = O.quantize(host(x))
    assert np.array_equal(host(s).astype(np.float32), want_s)
    assert np.array_equal(host(q), want_q)


MANY = [  # rows, groups, channels, columns: what the choice of a kernel goes by
    (1, 1, 4200, 4096), (3, 1, 40, 4160), (20, 1, 4112, 4160), (70, 1, 1000, 1024), (150, 1, 700, 1040), (90, 2, 300, 4224), (130, 40, 200, 192), (600, 40, 2100, 64),
    (1300, 40, 2050, 80), (3000, 40, 2050, 64), (4100, 40, 2050, 128), (7700, 40, 2050, 64), (400, 1, 8500, 64), (2600, 1, 5200, 64), (900, 20, 300, 4096),
]


@pytest.mark.parametrize("shape", MANY, ids=str)
def test_every_kernel(shape):
    announce(f"i8 {shape}")
    rows, groups, N, K = shape
    rng = np.random.default_rng(rows)
    cuts = np.sort(rng.integers(0, rows + 1, groups - 1)) if groups > 1 else None
    ptr = None if groups == 1 else [0, *cuts.tolist(), rows]
    check_product(i8(rng, rows, K), i8(rng, groups, N, K), ptr, "bf16", rng)


@pytest.mark.parametrize("groups", [63, 64, 255, 256, 511, 512, 513, 1100, 4096])
@pytest.mark.parametrize("columns", [64, 70])
def test_many_groups(groups, columns):
    """As many groups as lanes look for a tile, and one more or less; sizes that give tiles and few rows."""
    announce(f"i8 {groups} groups of {columns}")
    rng = np.random.default_rng(groups)
    for rows, N in ((groups // 3, 16), (40 * groups, 24)):
        lengths = rng.multinomial(rows, rng.dirichlet(np.full(groups, 0.3)))
        check_product(i8(rng, rows, columns), i8(rng, groups, N, columns), np.concatenate([[0], np.cumsum(lengths)]).tolist(), "f16", rng)


@pytest.mark.parametrize("steps", range(15))
@pytest.mark.parametrize("size", [(300, 500), (424, 13960), (3000, 4100)], ids=str)
def test_any_number_of_steps(size, steps):
    """Columns around every multiple of 64 that a round of the tiles' buffers may end at."""
    M, N = size
    rng = np.random.default_rng(steps)
    for K in (64 * steps + 16, 64 * steps + 48, 64 * steps + 64):
        announce(f"i8 steps {size} {K}")
        a, b = rng.integers(-127, 128, (M, K)).astype(np.int8), rng.integers(-127, 128, (N, K)).astype(np.int8)
        ones = torch.ones(max(M, N), device="cuda:0")
        got = S.seer_i8_product(torch.from_numpy(a).cuda(), ones[:M], torch.from_numpy(b).cuda()[None], ones[None, :N], dtype=torch.float32)
        want = a.astype(np.float32) @ b.astype(np.float32).T         # exact: below 2^24
        assert np.array_equal(got.cpu().numpy(), want)


PARTLY = [  # rows, channels, columns, how far the rows lie apart: rows at multiples of 16 that end within 16 bytes
    (1, 17, 1, 16), (3, 40, 15, 16), (5, 64, 17, 32), (1, 300, 4111, 4112), (40, 130, 1001, 1008), (70, 300, 63, 64), (130, 257, 65, 80),
    (500, 513, 259, 272), (700, 1025, 1023, 1040), (1000, 2049, 130, 144), (300, 200, 8191, 8192), (97, 16, 3089, 3104),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("shape", PARTLY, ids=str)
def test_rows_that_end_within_a_piece(shape, kind):
    """What lies between the rows' ends and the next multiple of 16 is anything, and has no part in the sums."""
    announce(f"i8 partly {shape} {kind}")
    M, N, K, ld = shape
    rng = np.random.default_rng(M + K)
    check_product(spread(i8(rng, M, K), ld, 99), spread(i8(rng, N, K), ld, -77)[None], None, kind, rng)
    lengths = rng.multinomial(M, [0.5, 0.1, 0.4])
    b = spread(i8(rng, 3 * N, K), ld, 55).unflatten(0, (3, N))
    check_product(spread(i8(rng, M, K), ld, 99), b, np.concatenate([[0], np.cumsum(lengths)]).tolist(), kind, rng)


SHARED = [  # rows, channels, columns: one product whose columns are shared out between workgroups
    (97, 16, 3088), (100, 300, 4112), (129, 257, 8192), (500, 130, 4112), (1000, 500, 6160), (300, 1001, 5136), (3000, 129, 8208),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("shape", SHARED, ids=str)
def test_shared_columns(shape, kind):
    announce(f"i8 shared {shape} {kind}")
    M, N, K = shape
    assert S.i8_product_workspace_bytes(M, N, K) > 0
    rng = np.random.default_rng(M + K)
    check_product(i8(rng, M, K), i8(rng, 1, N, K), None, kind, rng)


SHARED_GROUPS = [  # lengths of the groups, rows behind them, channels, columns
    ([300, 0, 64, 1, 130], 9, 100, 6672), ([0, 0, 77, 40], 0, 257, 8192), ([70] * 20, 3, 30, 4112), ([0] * 20 + [700, 1], 0, 64, 9216), ([300], 5, 60, 8192),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("groups", SHARED_GROUPS, ids=lambda g: f"{len(g[0])}x{sum(g[0])}+{g[1]}-{g[2]}-{g[3]}")
def test_shared_columns_of_groups(groups, kind):
    lengths, more, N, K = groups
    announce(f"i8 shared groups {lengths} {kind}")
    rng = np.random.default_rng(N + K)
    M = sum(lengths) + more
    assert S.i8_product_workspace_bytes(M, N, K, len(lengths)) > 0
    check_product(i8(rng, M, K), i8(rng, len(lengths), N, K), np.concatenate([[0], np.cumsum(lengths)]).tolist(), kind, rng)


def test_shared_columns_of_no_group_are_zero_whatever_they_hold():
    rng = np.random.default_rng(4)
    a, b, sa = i8(rng, 300, 8192), i8(rng, 3, 70, 8192), torch.full((300,), float("nan"), device="cuda:0")
    sa[:200] = 1
    assert S.i8_product_workspace_bytes(300, 70, 8192, 3) > 0
    y = S.seer_i8_product(a, sa, b, torch.ones(3, 70, device="cuda:0"), group_ptr=torch.tensor([0, 120, 120, 200], dtype=torch.int32, device="cuda:0"))
    assert not y[200:].any() and bool(torch.isfinite(y.float()).all())


def test_shared_columns_with_a_workspace_of_the_callers():
    rng = np.random.default_rng(8)
    M, N, K = 300, 200, 4096
    a, b = i8(rng, M, K), i8(rng, 1, N, K)
    sa, sb = torch.rand(M, device="cuda:0"), torch.rand(1, N, device="cuda:0")
    need = S.i8_product_workspace_bytes(M, N, K)
    want = S.seer_i8_product(a, sa, b, sb)
    ws = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda:0")
    assert torch.equal(S.seer_i8_product(a, sa, b, sb, workspace=ws[:need]), want)
    assert bool((ws[need:] == 255).all())
    with pytest.raises(S.SeerError):
        S.seer_i8_product(a, sa, b, sb, workspace=ws[: need - 1])
    ptr = torch.tensor([0, M], dtype=torch.int32, device="cuda:0")
    assert torch.equal(S.seer_i8_product(a, sa, b, sb, group_ptr=ptr), want)


@pytest.mark.parametrize("K", [16, 112, 128, 144, 256, 272, 640])
def test_tiles_that_end_in_one_row_and_one_channel(K):
    """Lines are fetched behind the columns' end, of a range that is one row long."""
    announce(f"i8 2817 x 1537 x {K}")
    rng = np.random.default_rng(K)
    a, b = i8(rng, 2817, K), i8(rng, 1, 1537, K)
    assert S.i8_product_kernel(a, b) == "tiles"
    check_product(a, b, None, "f32", rng)
