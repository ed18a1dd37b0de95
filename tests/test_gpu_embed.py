"""seer_embed and seer_embed_grad against their definitions."""
import numpy as np
import pytest
import torch

import paper_2403_17017_amd as S
from oracle import token_oracle as O
from tests.gpu_util import announce
from tests.routed_util import ROUND, TINY, TYPES, U32, assert_within, host, rounded, shifted, spread

pytestmark = pytest.mark.gpu
INDEX = {"i32": torch.int32, "i64": torch.int64}


def ids(values, index="i64"):
    return torch.from_numpy(np.asarray(values)).to(INDEX[index]).cuda()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("size", [(1, 1, 1), (1, 5, 4096), (7, 3, 64), (33, 1000, 1023), (300, 17, 8), (5, 100, 8192), (2, 9, 9001), (0, 5, 16), (4, 0, 8), (1025, 77, 130)], ids=str)
def test_lookup(size, kind):
    T, V, D = size
    announce(f"embed {size} {kind}")
    rng = np.random.default_rng(T + D)
    table = rounded(rng.standard_normal((V, D)), kind)
    token = rng.integers(-1, V + 2, T)
    if T > 4:
        token[1], token[2], token[3] = -(1 << 30), (1 << 31) - 1, V
    for scale in (1.0, 0.3, -64.0):
        f32 = float(np.float32(scale))
        want = O.embed(token, host(table), f32) if V else np.zeros((T, D))
        for index in INDEX:
            got = host(S.seer_embed(ids(token, index), table, scale=scale))
            if scale == 1.0:
                assert np.array_equal(got, want)
            else:
                assert_within(got, want, np.abs(want) * (ROUND[kind] + U32 * (kind != "f32")) * 1.01 + TINY[kind], "embed")


def test_lookup_of_bits_strides_and_far_numbers():
    rng = np.random.default_rng(2)
    table = torch.from_numpy(rng.integers(0, 1 << 16, (50, 33)).astype(np.uint16).view(np.int16)).cuda().view(torch.bfloat16)       # NaNs and all
    token = ids([[3, 49, -1], [0, 0, 1 << 40]])
    out = S.seer_embed(token, table)
    assert torch.equal(out[:2].view(torch.int16), table[[3, 49]].view(torch.int16)) and not out[[2, 5]].view(torch.int16).any()
    room = torch.full((6, 48), 55.0, dtype=torch.bfloat16, device="cuda:0")
    S.seer_embed(token, shifted(table, 1), out=room[:, :33])
    assert torch.equal(room[:, :33].contiguous().view(torch.int16), out.view(torch.int16)) and bool((room[:, 33:] == 55).all())
    for other in (spread(table, 40), spread(table, 64)):
        assert torch.equal(S.seer_embed(token, other).view(torch.int16), out.view(torch.int16))


def check_grad(token, dy, V, kind, grad, scale=1.0, accumulate=False, index="i64", **k):
    D = dy.shape[1]
    f32 = float(np.float32(scale))
    want, size, n = O.embed_grad(token, host(dy), V, f32)
    held = rounded(np.random.default_rng(1).standard_normal((V, D)), grad) if accumulate else None
    got = S.seer_embed_grad(ids(token, index), dy, V, scale=scale, accumulate=accumulate, dtype=TYPES[grad], dtable=held.clone() if accumulate else None, **k)
    assert got.dtype == TYPES[grad] and got.shape == (V, D)
    if accumulate:
        before = host(held)
        want, size = want + before, size + np.abs(before)
        assert torch.equal(got[torch.from_numpy(n[:, 0] == 0).cuda()], held[torch.from_numpy(n[:, 0] == 0).cuda()])
    # a unit for each addition, the product and its sum
    off = U32 * (n + 2) * size
    assert_within(host(got), want, off + (np.abs(want) + off) * ROUND[grad] + TINY[grad], "dtable")


GRADS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")]
SIZES = [  # tokens, rows, columns, skew
    (1, 1, 1, 0), (1, 9, 64, 0), (5, 3, 130, 0), (64, 64, 8, 1), (100, 7, 1023, 1), (1031, 1300, 33, 1), (300, 40000, 16, 0.5), (2500, 3, 48, 0), (4100, 1, 24, 0),
    (9000, 500, 16, 1), (3, 70, 4104, 0), (40, 2, 2056, 0), (0, 12, 40, 0), (8193, 70000, 8, 1.3), (20000, 11, 9, 0.3),
]


@pytest.mark.parametrize("accumulate", [False, True], ids=["", "add"])
@pytest.mark.parametrize("types", GRADS, ids=lambda t: f"{t[0]}-{t[1]}")
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradient(size, types, accumulate):
    T, V, D, skew = size
    announce(f"embed_grad {size} {types} {accumulate}")
    rng = np.random.default_rng(T + D)
    p = np.arange(1, V + 1) ** -float(skew)
    token = rng.choice(V, size=T, p=p / p.sum())
    if T > 8:
        token[rng.random(T) < 0.1] = -1
        token[3], token[4] = V, (1 << 31) - 1
    check_grad(token, rounded(rng.standard_normal((T, D)), types[0]), V, *types, scale=64.0 if T % 2 else 0.3, accumulate=accumulate, index="i32" if T % 3 else "i64")


@pytest.mark.parametrize("first", [0, 1, 31, 32, 33])
@pytest.mark.parametrize("many", [1, 30, 31, 32, 33, 63, 64, 65, 1023, 1024, 1025, 1056, 2048, 2081])
def test_one_row_of_many_tokens(many, first):
    """Where the runs that are summed beforehand begin and end within, at and beyond the row's places."""
    announce(f"embed_grad run {many} behind {first}")
    rng = np.random.default_rng(many)
    token = np.concatenate([np.zeros(first), np.ones(many), np.full(37, 2)]).astype(np.int64)
    check_grad(rng.permutation(token), rounded(rng.standard_normal((token.size, 12)), "f32"), 4, "f32", "f32")


def test_order_is_the_tokens():
    """Sums in fp32 of values of very different size: the same bits on every run, whatever else the row numbers are."""
    rng = np.random.default_rng(4)
    token = rng.integers(0, 20, 12000)
    dy = rounded(rng.standard_normal((12000, 40)) * 10.0 ** rng.integers(-6, 6, (12000, 1)), "f32")
    first = S.seer_embed_grad(ids(token), dy, 20)
    for _ in range(3):
        assert torch.equal(first, S.seer_embed_grad(ids(token), dy, 20))
    few = S.seer_embed_grad(ids(token[:5000]), dy[:5000].contiguous(), 20)
    wide = S.seer_embed_grad(ids(token[:5000] * 100000), dy[:5000].contiguous(), 2000000)
    assert torch.equal(few, wide[torch.arange(20, device="cuda:0") * 100000]) and int((wide != 0).any(1).sum()) == 20


def test_infinities_and_nan_stay_in_their_row():
    dy = torch.ones(6, 10, device="cuda:0")
    dy[1], dy[2, 3], dy[4] = float("nan"), float("inf"), float("nan")
    d = S.seer_embed_grad(ids([0, 1, 2, 2, -1, 5]), dy, 6, scale=2.0)
    assert bool((d[[0, 5]] == 2).all()) and bool(d[1].isnan().all()) and bool(d[2, 3].isinf()) and bool((d[2, 4:] == 4).all()) and not d[[3, 4]].any()
    d = S.seer_embed_grad(ids([0]), dy[:1], 3, scale=float("inf"))
    assert bool(d[0].isinf().all()) and not d[1:].any()              # rows that are no token's are zeros whatever the scale


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_strides_workspaces_and_what_lies_beside(kind):
    rng = np.random.default_rng(5)
    token = rng.integers(-1, 90, 3000)
    dy = rounded(rng.standard_normal((3000, 75)), kind)
    want = S.seer_embed_grad(ids(token), dy, 90)
    need = S.embed_grad_workspace_bytes(3000, 90, 75)
    ws = torch.full((need + 64,), 0xEE, dtype=torch.uint8, device="cuda:0")
    for other in (spread(dy, 80), shifted(dy, 1), spread(shifted(dy, 1), 101)):
        room = torch.full((90, 99), 55.0, dtype=dy.dtype, device="cuda:0")
        S.seer_embed_grad(ids(token), other, dtable=room[:, :75], workspace=ws[16: 16 + need])
        assert torch.equal(room[:, :75], want) and bool((room[:, 75:] == 55).all())
        assert bool((ws[:16] == 0xEE).all()) and bool((ws[16 + need:] == 0xEE).all())


def test_rows_and_columns_beyond_32_bits():
    """A table of 4.6 G elements: the last rows are looked up, and have a gradient."""
    announce("embedding beyond 2^32 elements")
    V, D = 1120000, 4096
    table = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda:0")
    far = torch.tensor([V - 1, 5, V - 2, 1100000, V - 1, 1048577], device="cuda:0")
    table[far] = torch.arange(1, 7, device="cuda:0")[:, None].to(torch.bfloat16)
    out = S.seer_embed(far, table, scale=2.0)
    assert torch.equal(out, 2 * table[far])
    d = S.seer_embed_grad(far, out, dtable=table)
    for column in (0, -1):          # (which of two assignments to a row of the table stays may differ from column to column)
        want = torch.zeros(V, device="cuda:0")
        want.index_add_(0, far, out[:, column].float())
        assert torch.equal(d[:, column].float(), want)


def test_on_another_stream_and_captured():
    announce("embedding captured")
    g = torch.Generator(device="cuda:0").manual_seed(3)
    table = torch.randn(500, 72, generator=g, device="cuda:0")
    for T in (300, 9000):
        token = torch.randint(-1, 500, (T,), generator=g, device="cuda:0")
        dy = torch.randn(T, 72, generator=g, device="cuda:0")
        want = [S.seer_embed(token, table, scale=3.0), S.seer_embed_grad(token, dy, 500, scale=3.0)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = [S.seer_embed(token, table, scale=3.0, stream=side), S.seer_embed_grad(token, dy, 500, scale=3.0, stream=side)]
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        out, ws = [torch.empty_like(t) for t in want], S.alloc_workspace(S.embed_grad_workspace_bytes(T, 500, 72))
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            S.seer_embed(token, table, scale=3.0, out=out[0])
            S.seer_embed_grad(token, dy, scale=3.0, dtable=out[1], workspace=ws)
        for k in range(4):
            token.copy_(torch.randint(-1, 500, (T,), generator=g, device="cuda:0"))
            for t in out:
                t.fill_(7)
            ws.fill_(k)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[0], S.seer_embed(token, table, scale=3.0)) and torch.equal(out[1], S.seer_embed_grad(token, dy, 500, scale=3.0))


@pytest.mark.parametrize("V", [3, 5000, 1500000])
def test_more_tokens_than_one_pass_of_workgroups(V):
    """300 000 tokens, a third of them one row's: shares of the sort longer than a wave, and sums of sums of sums."""
    announce(f"300 000 tokens of {V}")
    g = torch.Generator(device="cuda:0").manual_seed(6)
    token = torch.randint(-1, V, (300000,), generator=g, device="cuda:0")
    token[torch.rand(300000, generator=g, device="cuda:0") < 0.33] = 1
    dy = torch.randn(300000, 8, generator=g, device="cuda:0")
    got = S.seer_embed_grad(token, dy, V, scale=0.5)
    known = token >= 0
    at, rows = token[known], dy[known].double()
    want = torch.zeros(V, 8, dtype=torch.float64, device="cuda:0").index_add_(0, at, rows) * 0.5
    size = torch.zeros(V, 8, dtype=torch.float64, device="cuda:0").index_add_(0, at, rows.abs()) * 0.5
    # runs of 16, of these 16, and what is left: no element goes through more than 16 + 16 + 2^17 / 256 + 62 additions
    assert bool(((got - want).abs() <= U32 * 700 * size + U32 * want.abs()).all())
    assert torch.equal(got, S.seer_embed_grad(token.int(), dy, V, scale=0.5))


@pytest.mark.parametrize("accumulate", [False, True], ids=["", "add"])
@pytest.mark.parametrize("types", GRADS, ids=lambda t: f"{t[0]}-{t[1]}")
@pytest.mark.parametrize("size", [(4097, 512, 24, 0.5), (9000, 1000, 16, 1), (5000, 1023, 130, 0), (9000, 1 << 18, 8, 0.8), (20000, (1 << 20) - 1, 4, 0)], ids=str)
def test_gradient_by_digits_of_ten_bits(size, types, accumulate):
    """More than 4096 tokens of tables of 512 to 1023 rows, and of 2^18 to 2^20 - 1: places are counted in 1024 buckets a wave."""
    T, V, D, skew = size
    announce(f"embed_grad ten bits {size} {types} {accumulate}")
    rng = np.random.default_rng(T + V)
    p = np.arange(1, V + 1) ** -float(skew)
    token = rng.choice(V, size=T, p=p / p.sum())
    token[rng.random(T) < 0.05] = -1
    token[5], token[6], token[7] = V, V - 1, 0
    check_grad(token, rounded(rng.standard_normal((T, D)), types[0]), V, *types, scale=0.3, accumulate=accumulate, index="i32" if T % 3 else "i64")
