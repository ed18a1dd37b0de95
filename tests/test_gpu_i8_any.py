"""seer_i8_product where rows do not lie at multiples of 16 bytes, in sizes that go to the tiled kernel for any address."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2403_17017_amd as S
from paper_2403_17017_amd import routed as R
from tests.gpu_util import announce
from tests.routed_util import TYPES, shifted, spread
from tests.test_gpu_i8_product import check_product, i8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("columns", [1, 15, 17, 33, 100, 111, 113, 127])
def test_fewer_columns_than_a_step(columns, kind):
    """Pieces behind the end of a row that is shorter than the 128 columns of a step."""
    announce(f"i8 any, {columns} columns, {kind}")
    rng = np.random.default_rng(columns)
    for M, N in ((300, 300), (1000, 1000), (641, 129)):
        check_product(spread(i8(rng, M, columns), columns + 1, 99), spread(i8(rng, N, columns), columns + 2, -77)[None], None, kind, rng)
    lengths = [700, 0, 1, 129, 513, 300, 255, 102]
    a, b = shifted(i8(rng, sum(lengths) + 37, columns), 1), shifted(i8(rng, 8, 256, columns), 3)
    check_product(a, b, np.concatenate([[0], np.cumsum(lengths)]).tolist(), kind, rng)


def apart(t, where, by):
    """The matrix with its rows off multiples of 16 bytes: their distance, the first one's address, or both."""
    ld = t.shape[-1] + (by if where != "shifted" else 0)
    ld += ld % 16 == 0 and where != "shifted"
    room = torch.full((t.shape[0] * ld + 64,), 99, dtype=torch.int8, device="cuda:0")
    start = by if where != "apart" else 0
    view = room.as_strided(t.shape, (ld, 1), start)
    view.copy_(t)
    return view


ANY = [  # rows, channels, columns: off 128 in every size, with whole steps and without
    (300, 300, 100), (257, 511, 129), (1000, 333, 255), (700, 777, 384), (2001, 130, 511), (300, 2049, 640), (3001, 700, 1027),
]


@pytest.mark.parametrize("by", [1, 2, 3, 5])
@pytest.mark.parametrize("where", ["apart", "shifted", "both"])
@pytest.mark.parametrize("shape", ANY, ids=str)
def test_any_address(shape, where, by):
    """Values of which no two rows or columns are alike, at every remainder of an address."""
    M, N, K = shape
    announce(f"i8 any {shape} {where} {by}")
    rng = np.random.default_rng(M + K + by)
    a, b = i8(rng, M, K), i8(rng, N, K)
    for x, y in ((apart(a, where, by), b), (a, apart(b, where, by)), (apart(a, where, by), apart(b, where, 4 - by % 4))):
        assert S.i8_product_kernel(x, y) == "any" or (x.data_ptr() | y.data_ptr() | x.stride(0) | y.stride(0)) % 16 == 0
        check_product(x, y[None], None, "bf16" if by % 2 else "f32", rng)


ANY_GROUPS = [  # lengths of the groups, rows behind them, channels, columns
    ([300, 0, 129, 1, 640, 70], 11, 130, 129), ([128, 256, 384, 1], 0, 257, 513), ([0, 0, 2000, 0], 3, 300, 100), ([255, 257, 127, 511], 130, 513, 1041),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("groups", ANY_GROUPS, ids=lambda g: f"{len(g[0])}x{sum(g[0])}+{g[1]}-{g[2]}-{g[3]}")
def test_groups_at_any_address(groups, kind):
    lengths, more, N, K = groups
    announce(f"i8 any groups {lengths} {kind}")
    rng = np.random.default_rng(N + K)
    M, G = sum(lengths) + more, len(lengths)
    ptr = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    for by in (1, 2, 3):
        a, b = apart(i8(rng, M, K), "both", by), apart(i8(rng, G * N, K), "both", 4 - by).unflatten(0, (G, N))
        assert S.i8_product_kernel(a, b, torch.tensor(ptr, dtype=torch.int32)) == "any"
        check_product(a, b, ptr, kind, rng)


@pytest.mark.parametrize("shape", [(97, 16, 3089), (500, 130, 4111), (100, 512, 8190)], ids=str)
def test_long_columns_without_a_workspace(shape):
    """Sizes at which aligned rows would need a workspace: neither kernel for others does."""
    M, N, K = shape
    announce(f"i8 any without a workspace {shape}")
    rng = np.random.default_rng(K)
    a, b = apart(i8(rng, M, K), "both", 1), apart(i8(rng, N, K), "both", 3)
    assert S.i8_product_workspace_bytes(M, N, K) > 0 and S.i8_product_kernel(a, b) in ("any", "few")
    check_product(a, b[None], None, "f32", rng)
    out, ones = torch.full((M, N), float("nan"), device="cuda:0"), torch.ones(max(M, N), device="cuda:0")
    d = lambda t, kind: C.byref(R.seer_dense(t.data_ptr(), t.shape[0], t.shape[1], t.stride(0), kind))
    stream = torch.cuda.current_stream().cuda_stream
    assert S.lib().seer_i8_product(d(a, 3), ones.data_ptr(), d(b, 3), ones.data_ptr(), None, 1, d(out, 0), None, 0, stream) == 0
    want = a.cpu().to(torch.int32).numpy().astype(np.int64) @ b.cpu().to(torch.int32).numpy().astype(np.int64).T
    assert np.array_equal(out.cpu().numpy(), want.astype(np.float32))
