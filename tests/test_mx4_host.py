"""CPU-only tests of rows in 4-bit floating point: the refusal of bad arguments before any launch, and pins of the oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2403_17017_amd as S
from oracle import routed_oracle as O
from paper_2403_17017_amd import mx4 as M
from paper_2403_17017_amd import routed as R
from tests.marshal_util import Described, DescribedRouting
from tests.test_routed_host import dense, routing

EINVAL, EWORKSPACE, ELIMIT = -1, -4, -6
A, B_, D_, W, P = 1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20       # addresses that nothing reads: every call below is refused or empty
FAR = 1 << 40


def mx4(data, scale, rows, cols, ld=None, scale_ld=None):
    blocks = -(-cols // 32)
    return C.byref(M.seer_mx4(data, scale, rows, cols, 16 * blocks if ld is None else ld, blocks if scale_ld is None else scale_ld))


def test_layout():
    assert C.sizeof(M.seer_mx4) == 48 and M.seer_mx4.rows.offset == 16


def test_quantise_refusals():
    f = S.lib().seer_mx4_quantize
    x = dense(A, 4, 40)

    def call(x=x, q=mx4(B_, W, 4, 40)):
        return f(x, q, None)
    assert call(x=None) == EINVAL and call(q=None) == EINVAL and call(x=dense(A, 4, 40, kind=3)) == EINVAL and call(x=dense(A, 4, 41)) == EINVAL
    assert call(q=mx4(B_, W, 5, 40)) == EINVAL and call(q=mx4(B_, W, 4, 40, ld=16)) == EINVAL and call(q=mx4(B_, W, 4, 40, ld=40)) == EINVAL
    assert call(q=mx4(B_, W, 4, 40, scale_ld=1)) == EINVAL and call(q=mx4(B_ + 8, W, 4, 40)) == EINVAL and call(q=mx4(None, W, 4, 40)) == EINVAL
    assert call(q=mx4(B_, None, 4, 40)) == EINVAL and call(q=mx4(A, W, 4, 40)) == EINVAL and call(q=mx4(B_, A + 100, 4, 40)) == EINVAL
    assert call(q=mx4(B_, B_ + 127, 4, 40)) == EINVAL                    # scales over the last code
    assert call(q=mx4(B_, W, 4, 40, ld=1 << 62)) == EINVAL
    assert call(x=dense(None, 0, 40), q=mx4(None, None, 0, 40)) == 0 and call(x=dense(None, 4, 0), q=mx4(None, None, 4, 0)) == 0
    g = S.lib().seer_route_gather_mx4
    to = mx4(B_, W, 8, 40)
    assert g(None, x, to, None) == EINVAL and g(routing(), None, to, None) == EINVAL and g(routing(), x, mx4(B_, W, 4, 40), None) == EINVAL
    assert g(routing(slots=W - 16), x, to, None) == EINVAL and g(routing(slots=B_ + 64), x, to, None) == EINVAL and g(routing(experts=5000), x, to, None) == ELIMIT


def test_product_refusals():
    f = S.lib().seer_mx4_product

    def call(a=mx4(A, A + 4096, 4, 64), b=mx4(B_, B_ + 4096, 16, 64), ptr=P, groups=2, out=dense(D_, 4, 8, kind=1), ws=None, size=0):
        return f(a, b, ptr, groups, out, ws, size, None)
    assert call(a=None) == EINVAL and call(b=None) == EINVAL and call(out=None) == EINVAL and call(groups=0) == EINVAL and call(ptr=None) == EINVAL
    assert call(ptr=P + 2) == EINVAL and call(groups=3) == EINVAL and call(a=mx4(A, A + 4096, 4, 96)) == EINVAL and call(a=mx4(A + 4, A + 4096, 4, 64)) == EINVAL
    assert call(b=mx4(B_, B_ + 4096, 16, 64, ld=24)) == EINVAL and call(out=dense(D_, 5, 8, kind=1)) == EINVAL and call(out=dense(D_, 4, 8, kind=3)) == EINVAL
    for at in (A, A + 4096, B_, B_ + 4096, P):
        assert call(out=dense(at, 4, 8, kind=1)) == EINVAL, at
    assert call(groups=4097, b=mx4(B_, 1 << 30, 4097 * 8, 64)) == ELIMIT
    assert call(a=mx4(None, None, 0, 64), out=dense(None, 0, 8, kind=1)) == 0
    assert S.mx4_product_workspace_bytes(-1, 4, 4) == S.mx4_product_workspace_bytes(4, 4, 4, 0) == 0


def test_what_the_binding_refuses(monkeypatch):
    monkeypatch.setattr(torch.cuda, "_initialized", True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    u8 = torch.uint8
    t = lambda shape, at, dtype=u8, **k: Described(shape, dtype, at * FAR, **k)
    x = lambda **k: t((4, 40), 1, torch.float32, **k)
    quantise = lambda x=x(), q=t((4, 32), 2), scale=t((4, 2), 3): S.seer_mx4_quantize(x, q=q, scale=scale, stream=0)
    with pytest.raises(RuntimeError, match="history"):
        quantise(x(requires_grad=True))
    with pytest.raises(TypeError):
        quantise(q=t((4, 32), 2, torch.int8))
    for bad in ({"q": t((4, 48), 2)}, {"q": t((4, 16), 2), "scale": t((4, 1), 3)}, {"scale": t((4, 3), 3)}, {"scale": t((5, 2), 3)}, {"scale": t((4, 2), 3, stride=(4, 2))},
                {"q": t((4, 32), 2, device=1)}, {"scale": t((4, 2), 3, device=-1)}):
        with pytest.raises(ValueError):
            quantise(**bad)
    with pytest.raises(S.SeerError):
        quantise(q=t((4, 32), 1))
    with pytest.raises(S.SeerError):
        S.seer_route_gather_mx4(DescribedRouting(4, 2, 3, 9 * FAR), x(), q=t((7, 32), 2), scale=t((7, 2), 3), stream=0)
    f32 = torch.float32
    product = lambda **k: S.seer_mx4_product(**{"a": t((4, 32), 1), "a_scale": t((4, 2), 2), "b": t((3, 8, 32), 3), "b_scale": t((3, 8, 2), 4),
                                                 "group_ptr": t((4,), 5, torch.int32), "out": t((4, 8), 6, f32), "stream": 0, **k})
    for bad in ({"a_scale": t((4, 3), 2)}, {"b_scale": t((24, 2), 4)}, {"b_scale": t((8, 3, 2), 4)}, {"group_ptr": t((3,), 5, torch.int32)}, {"b": t((3, 8, 32), 3, device=1)},
                {"workspace": t((64,), 7, device=-1)}):
        with pytest.raises(ValueError):
            product(**bad)
    for bad in ({"a": t((4, 32), 1, torch.int8)}, {"b_scale": t((3, 8, 2), 4, f32)}, {"dtype": torch.float16}):
        with pytest.raises(TypeError):
            product(**bad)
    with pytest.raises(S.SeerError):
        product(out=t((4, 8), 1, f32))
    with pytest.raises(S.SeerError):
        product(out=t((4, 9), 6, f32))


def test_oracle_pins():
    codes, scale = O.mx4_quantize(np.array([[6.0, 5, 2.5, -1.25, 0.25, 0.75, 7.9, -0.0] + [0] * 25 + [3e-3]]))
    assert scale.tolist() == [[127, 116]]
    assert O.mx4_values(codes, scale)[0, :8].tolist() == [6, 4, 2, -1, 0, 1, 6, 0] and codes[0, 0] == 0x67 and codes[0, 3] == 0x87
    assert np.isclose(O.mx4_values(codes, scale)[0, 33], 3e-3, rtol=0.07) and codes.shape == (1, 32)
    codes, scale = O.mx4_quantize(np.array([[np.inf, 1], [np.nan, 1], [2.0 ** -149, 0], [0, 0]]))
    assert scale.ravel().tolist() == [255, 255, 0, 0] and not codes.any()
    out, size = O.mx4_product(np.array([[1.0, -2], [3, 4], [5, 6]]), np.array([[[1.0, 1]], [[0, 1]]]), [0, 1, 2])
    assert out.ravel().tolist() == [-1, 4, 0] and size.ravel().tolist() == [3, 4, 0]


def kernel(rows, channels, columns, groups=1, ld=None, ptr=None):
    f = lambda at, n: C.byref(M.seer_mx4(at, at + 4096, n, columns, ld or 16 * -(-columns // 32), -(-columns // 32)))
    rc = S.lib().seer_mx4_product_kernel(f(A, rows), f(1 << 30, groups * channels), P if groups > 1 else ptr, groups)
    return S.MX4_KERNELS[rc] if rc >= 0 else rc


def test_kernels():
    assert kernel(1, 8192, 8192) == "few" and kernel(256, 2048, 4096, groups=64) == "few" and kernel(5, 6, 0) == "few"
    assert kernel(3001, 5001, 4111) == "tiles" and kernel(32768, 4096, 4096, groups=32) == "tiles"
    assert kernel(300, 512, 8192) == "shared" and S.mx4_product_workspace_bytes(300, 512, 8192) > 0
    assert kernel(3000, 5000, 4096, ld=1 << 23) == kernel(1, 5000, 4096, ld=1 << 23) == "any"      # too far apart for 32-bit offsets into a tile
    assert kernel(0, 5, 64) == kernel(5, 0, 64) == "none"
    # 2^30 tiles of 128 rows by 128 channels are too many for 32-bit numbers of tiles
    assert kernel(1 << 22, 1 << 22, 32) == -6 and kernel((1 << 22) - 1024, (1 << 22) - 1024, 32) in S.MX4_KERNELS
    assert kernel(4, 8, 64, groups=4097) == -6 and kernel(4, 8, 64, groups=0) == -1 and kernel(4, 8, 64, ld=24) == -1


def test_kernel_query_refusals():
    f = S.lib().seer_mx4_product_kernel
    assert f(None, mx4(B_, W, 8, 64), None, 1) == -1 and f(mx4(A, W, 4, 64), None, None, 1) == -1 and f(mx4(A, W, 4, 64), mx4(B_, W, 9, 64), P, 2) == -1
    assert f(mx4(A, W, 4, 64), mx4(B_, W, 8, 64), None, 2) == -1 and f(mx4(A, W, 4, 64), mx4(B_, W, 8, 96), None, 1) == -1
    with pytest.raises(ValueError):
        S.mx4_product_kernel(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(64, dtype=torch.uint8))
    assert S.mx4_product_kernel(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(2, 8, 64, dtype=torch.uint8), torch.zeros(3, dtype=torch.int32)) == "few"


def test_what_is_chosen_is_near_the_best():
    """Of 220 drawn sizes with every kernel timed."""
    import csv
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "profiles", "mx4_kernel_times.csv")
    with open(path) as f:
        rows = list(csv.DictReader(line for line in f if not line.startswith("#")))
    assert len(rows) == 220
    over = []
    for r in rows:
        times = {k: float(r[k]) for k in ("few", "tiles_64", "tiles_128", "tiles_256", "shared") if float(r[k]) > 0}
        kind = kernel(int(r["rows"]), int(r["channels"]), int(r["columns"]), int(r["groups"]))
        over.append(min(t for k, t in times.items() if k.startswith(kind)) / min(times.values()))
    assert np.mean(over) < 1.03 and max(over) < 1.6


def plan(rows, channels, columns, groups=1):
    f = lambda at, n: C.byref(M.seer_mx4(at, at + 4096, n, columns, 16 * -(-columns // 32), -(-columns // 32)))
    tokens, shares = C.c_int32(-7), C.c_int32(-7)
    rc = S.lib().seer_mx4_product_plan(f(A, rows), f(1 << 30, groups * channels), P if groups > 1 else None, groups, C.byref(tokens), C.byref(shares))
    return (S.MX4_KERNELS[rc] if rc >= 0 else rc), tokens.value, shares.value


def test_plans():
    assert plan(1, 8192, 8192) == ("few", 0, 1) and plan(0, 5, 64) == ("none", 0, 1) and plan(5, 6, 0) == ("few", 0, 1)
    assert plan(1000, 3001, 4096) == ("tiles", 64, 1) and plan(2817, 1537, 4096) == ("tiles", 128, 1) and plan(3001, 5001, 4111) == ("tiles", 256, 1)
    assert plan(32768, 4096, 4096, 32) == ("tiles", 256, 1)
    kind, tokens, shares = plan(300, 512, 8192)
    assert kind == "shared" and tokens == 64 and shares > 1 and shares * 300 * 512 * 4 <= S.mx4_product_workspace_bytes(300, 512, 8192)
    assert plan(1 << 22, 1 << 22, 32) == (-6, -7, -7) and plan(4, 8, 64, 4097) == (-6, -7, -7)      # nothing is written on error
    f = S.lib().seer_mx4_product_plan
    assert f(mx4(A, W, 2817, 64), mx4(B_, W, 1537, 64), None, 1, None, None) == S.MX4_KERNELS.index("tiles")
    assert f(None, mx4(B_, W, 8, 64), None, 1, None, None) == -1 and f(mx4(A, W, 4, 64), mx4(B_, W, 9, 64), P, 2, None, None) == -1
    assert S.mx4_product_plan(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(2, 8, 64, dtype=torch.uint8), torch.zeros(3, dtype=torch.int32)) == ("few", 0, 1)
    with pytest.raises(ValueError):
        S.mx4_product_plan(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(64, dtype=torch.uint8))


def test_shares_are_whole_rounds():
    """No share of the columns is empty, and each but the last has as many rounds of 16 blocks."""
    seen = set()
    for rows in (70, 130, 200, 300):
        for channels in (256, 300, 512, 700):
            for blocks in range(33, 700, 13):
                kind, tokens, shares = plan(rows, channels, 32 * blocks)
                if kind == "shared":
                    rounds = -(-blocks // 16)
                    each = -(-rounds // shares)
                    assert (shares - 1) * each < rounds <= shares * each
                    seen.add(shares)
    assert len(seen) > 3


def test_tiles_that_are_chosen_are_near_the_best():
    """Of the 220 sizes the very tiles that are planned, and as many shares as are planned where those were timed."""
    import csv
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "profiles", "mx4_kernel_times.csv")
    with open(path) as f:
        rows = list(csv.DictReader(line for line in f if not line.startswith("#")))
    over, kinds = [], set()
    for r in rows:
        times = {k: float(r[k]) for k in ("few", "tiles_64", "tiles_128", "tiles_256", "shared") if float(r[k]) > 0}
        kind, tokens, shares = plan(int(r["rows"]), int(r["channels"]), int(r["columns"]), int(r["groups"]))
        kinds.add((kind, tokens))
        # (of shares the best are timed; another number of them counts with what the library's choice took)
        took = times[f"tiles_{tokens}"] if kind == "tiles" else times["few"] if kind == "few" else times["shared"] if shares == int(r["shares"]) else float(r["chosen"])
        over.append(took / min(times.values()))
    assert kinds == {("few", 0), ("tiles", 64), ("tiles", 128), ("tiles", 256), ("shared", 64)}
    assert np.mean(over) < 1.03 and max(over) < 1.6
