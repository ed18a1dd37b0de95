"""CPU-only tests of the router's choice and of the embedding: the refusal of bad arguments before any launch, and pins of the
oracle that the GPU tests go by."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2403_17017_amd as S
from oracle import token_oracle as O
from paper_2403_17017_amd import routed as R
from paper_2403_17017_amd import router
from tests.marshal_util import Described

EINVAL, EWORKSPACE, ELIMIT = -1, -4, -6
A, B_, D_, W, P = 1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20       # addresses that nothing reads: every call below is refused or empty
FAR = 1 << 40


def dense(data, rows, cols, ld=None, kind=0):
    return C.byref(R.seer_dense(data, rows, cols, cols if ld is None else ld, kind))


def how(choices=2, score=0, groups=1, best=1, group_best=1, renormalise=1, factor=1.0):
    return C.byref(router.seer_choice(choices, score, groups, best, group_best, renormalise, factor))


def test_layout():
    assert C.sizeof(router.seer_choice) == 28 and router.seer_choice.factor.offset == 24


def test_choose_refusals():
    f = S.lib().seer_route_choose

    def call(x=dense(A, 4, 8), bias=None, h=how(), expert=W, weight=P):
        return f(x, bias, h, expert, weight, None)
    assert call(x=None) == EINVAL and call(h=None) == EINVAL and call(expert=None) == EINVAL and call(weight=None) == EINVAL
    assert call(x=dense(A, 4, 8, 7)) == EINVAL and call(x=dense(A, 4, 8, kind=3)) == EINVAL and call(x=dense(None, 4, 8)) == EINVAL
    assert call(x=dense(A, 4, 0)) == EINVAL and call(x=dense(A, 4, 4097)) == ELIMIT
    for k in ({"choices": 0}, {"choices": 9}, {"score": 2}, {"groups": 0}, {"groups": 3}, {"groups": 2, "best": 3}, {"best": 0}, {"group_best": 3},
              {"groups": 4, "best": 1, "choices": 3}, {"factor": float("inf")}, {"factor": float("nan")}):
        assert call(h=how(**k)) == EINVAL, k
    assert call(x=dense(A, 4, 130), h=how(choices=65)) == ELIMIT and call(x=dense(A, 4, 130), h=how(groups=65)) == ELIMIT
    assert call(bias=6) == EINVAL and call(expert=W + 2) == EINVAL and call(weight=P + 1) == EINVAL
    assert call(weight=W + 28) == EINVAL and call(expert=A + 124) == EINVAL and call(weight=A) == EINVAL and call(bias=W) == EINVAL and call(bias=P + 28) == EINVAL
    assert call(x=dense(A, (1 << 31) - 1, 8), h=how(choices=2)) == EINVAL
    assert call(x=dense(None, 0, 8), expert=None, weight=None) == 0
    g = S.lib().seer_route_choose_grad

    def back(x=dense(A, 4, 8), h=how(), expert=W, dweight=P, to=dense(B_, 4, 8)):
        return g(x, h, expert, dweight, to, None)
    assert back(x=None) == EINVAL and back(h=None) == EINVAL and back(expert=None) == EINVAL and back(dweight=None) == EINVAL and back(to=None) == EINVAL
    assert back(to=dense(B_, 4, 7)) == EINVAL and back(to=dense(B_, 4, 8, kind=1)) == EINVAL and back(to=dense(A, 4, 8)) == EINVAL
    assert back(to=dense(W, 4, 8)) == EINVAL and back(to=dense(P - 96, 4, 8)) == EINVAL and back(h=how(choices=0)) == EINVAL
    assert back(x=dense(None, 0, 8), to=dense(None, 0, 8), expert=None, dweight=None) == 0


def test_embed_refusals():
    L = S.lib()

    def call(token=W, kind=5, table=dense(A, 100, 8), out=dense(B_, 4, 8)):
        return L.seer_embed(token, kind, table, 1.0, out, None)
    assert call(table=None) == EINVAL and call(out=None) == EINVAL and call(token=None) == EINVAL and call(token=W + 4) == EINVAL and call(kind=0) == EINVAL
    assert call(out=dense(B_, 4, 7)) == EINVAL and call(out=dense(B_, 4, 8, kind=1)) == EINVAL and call(table=dense(A, 100, 8, kind=3)) == EINVAL
    assert call(out=dense(A + 3200 - 32, 4, 8)) == EINVAL and call(out=dense(W, 4, 8)) == EINVAL
    assert call(token=None, out=dense(None, 0, 8)) == 0 and call(table=dense(None, 100, 0), out=dense(None, 4, 0)) == 0

    def back(token=W, kind=5, dy=dense(A, 4, 8, kind=1), add=0, to=dense(B_, 100, 8, kind=1), ws=P, size=1 << 20):
        return L.seer_embed_grad(token, kind, dy, 1.0, add, to, ws, size, None)
    assert back(dy=None) == EINVAL and back(to=None) == EINVAL and back(token=None) == EINVAL and back(kind=4, token=W + 2) == EINVAL and back(kind=1) == EINVAL
    assert back(to=dense(B_, 100, 9, kind=1)) == EINVAL and back(to=dense(B_, 100, 8, kind=2)) == EINVAL and back(to=dense(A, 100, 8, kind=1)) == EINVAL
    assert back(to=dense(W - 160, 100, 8, kind=1)) == EINVAL and back(dy=dense(A, 4, 8), to=dense(B_, 100, 8, kind=1)) == EINVAL
    assert back(ws=None) == EWORKSPACE and back(ws=P + 8) == EWORKSPACE and back(size=S.embed_grad_workspace_bytes(4, 100, 8) - 1) == EWORKSPACE
    assert back(ws=A) == EINVAL and back(ws=B_) == EINVAL and back(ws=W - 64) == EINVAL
    assert back(to=dense(None, 0, 8, kind=1)) == 0 and back(add=1, dy=dense(None, 0, 8, kind=1), token=None) == 0
    for tokens, rows, columns in ((0, 5, 5), (0, 0, 0), (1, 1, 1), (4097, 7, 0), ((1 << 31) - 1, (1 << 31) - 1, 1)):
        assert S.embed_grad_workspace_bytes(tokens, rows, columns) >= 16 * tokens + 8 * rows
    assert S.embed_grad_workspace_bytes(-1, 4, 4) == S.embed_grad_workspace_bytes(4, 1 << 31, 4) == 0


def test_what_the_binding_refuses(monkeypatch):
    monkeypatch.setattr(torch.cuda, "_initialized", True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    t = lambda shape, at, dtype=torch.float32, **k: Described(shape, dtype, at * FAR, **k)
    i32, i64 = torch.int32, torch.int64
    h = S.Choice(2)
    choose = lambda x=t((4, 8), 1), **k: S.seer_route_choose(x, h, **{"expert": t((4, 2), 2, i32), "weight": t((4, 2), 3), "stream": 0, **k})
    with pytest.raises(RuntimeError, match="history"):
        choose(t((4, 8), 1, requires_grad=True))
    for bad in ({"expert": t((4, 2), 2, i64)}, {"weight": t((4, 3), 3)}, {"bias": t((7,), 4)}, {"bias": t((8,), 4, stride=(2,))}, {"bias": t((8,), 4, device=1)},
                {"x": t((4, 8), 1, stride=(16, 2))}, {"x": t((4, 8), 1, device=-1)}, {"x": t((8,), 1)}, {"expert": t((4, 2), 2, i32, device=1)}):
        with pytest.raises(ValueError):
            choose(**bad)
    with pytest.raises(S.SeerError):
        choose(weight=t((4, 2), 2))                                  # on top of one another: the library's own
    with pytest.raises(ValueError):
        S.Choice(2, score="tanh")
    back = lambda expert=t((4, 2), 2, i32), dw=t((4, 2), 3), to=t((4, 8), 4): S.seer_route_choose_grad(t((4, 8), 1), h, expert, dw, dlogits=to, stream=0)
    for bad in ({"expert": t((4, 2), 2, i64)}, {"dw": t((4, 2), 3, torch.bfloat16)}, {"expert": None}, {"dw": None}):
        with pytest.raises(ValueError):
            back(**bad)
    with pytest.raises(S.SeerError):
        back(to=t((4, 8), 1))
    look = lambda token=t((4,), 1, i64), table=t((9, 8), 2), out=t((4, 8), 3): S.seer_embed(token, table, out=out, stream=0)
    for bad in ({"token": t((4,), 1)}, {"token": t((5,), 1, i64)}, {"token": t((4,), 1, i64, stride=(2,))}, {"token": None}, {"table": t((9, 8), 2, device=1)}):
        with pytest.raises(ValueError):
            look(**bad)
    with pytest.raises(RuntimeError, match="history"):
        look(table=t((9, 8), 2, requires_grad=True))
    with pytest.raises(S.SeerError):
        look(out=t((4, 8), 2))
    grad = lambda **k: S.seer_embed_grad(**{"token": t((4,), 1, i64), "dy": t((4, 8), 2), "dtable": t((9, 8), 3), "workspace": t((1 << 16,), 4, torch.uint8), "stream": 0, **k})
    for bad in ({"rows": 8}, {"dtype": torch.float16}, {"dtable": None}, {"dtable": None, "rows": 9, "accumulate": True}, {"token": t((4,), 1)},
                {"workspace": t((1 << 16,), 4, torch.uint8, device=1)}, {"token": t((3,), 1, i64)}):
        with pytest.raises(ValueError):
            grad(**bad)
    with pytest.raises(S.SeerError):
        grad(workspace=t((16,), 4, torch.uint8))
    with pytest.raises(S.SeerError):
        grad(dtable=t((9, 8), 2))


def test_oracle_pins():
    x = np.log(np.array([[1.0, 2.0, 3.0, 2.0]]))
    e, w = O.choose(x, 2)
    assert e.tolist() == [[2, 1]] and np.allclose(w, [[0.6, 0.4]])
    e, w = O.choose(x, 2, renormalise=False, factor=2.0)
    assert np.allclose(w, [[0.75, 0.5]])
    e, w = O.choose(x, 2, bias=[0.5, 0, 0, 0.1], renormalise=False)
    assert e.tolist() == [[0, 2]] and np.allclose(w, [[0.125, 0.375]])     # the bias chooses, the score weighs
    e, _ = O.choose([[5.0, 0, 4, 4]], 2, groups=2, best_groups=1)
    assert e.tolist() == [[0, 1]]
    e, _ = O.choose([[5.0, 0, 4, 4]], 2, score="sigmoid", groups=2, best_groups=1, group_best=2)
    assert e.tolist() == [[2, 3]]
    e, w = O.choose([[-np.inf, 1.0], [-np.inf, -np.inf]], 2, score="sigmoid")
    assert e.tolist() == [[1, -1], [-1, -1]] and np.allclose(w, [[1, 0], [0, 0]])
    e, w = O.choose([[-800.0, -801.0]], 2, score="sigmoid")
    assert np.allclose(w, [[1 / (1 + np.exp(-1)), 1 / (1 + np.exp(1))]])
    e, w = O.choose([[1.0, np.nan, 2]], 2)
    assert e.tolist() == [[1, 2]] and np.isnan(w).all()
    assert O.embed([1, -1, 3], np.array([[1.0], [2], [3]]), 2.0).ravel().tolist() == [4, 0, 0]
    d, size, n = O.embed_grad([1, 1, 5, -1], np.array([[1.0], [-3], [7], [9]]), 3, 2.0)
    assert d.ravel().tolist() == [0, -4, 0] and size.ravel().tolist() == [0, 8, 0] and n.ravel().tolist() == [0, 2, 0]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_oracle_gradient_by_differences(score, renormalise):
    """Central differences with a step of 1e-6 in 64 bits: off by some 1e-10."""
    rng = np.random.default_rng(3)
    x, dw = rng.standard_normal((3, 7)) * 2, rng.standard_normal((3, 3))
    x[1, 2] = -np.inf
    expert, _ = O.choose(x, 3, score=score, renormalise=renormalise, factor=1.5)
    got, _ = O.choose_grad(x, expert, dw, score, renormalise, 1.5)

    def value(x):                       # of the same experts
        s, _ = O.scores(x, score)
        w = np.take_along_axis(s, expert, 1)
        return float((1.5 * (w / w.sum(1, keepdims=True) if renormalise else w) * dw).sum())
    for t in range(3):
        for e in range(7):
            if np.isinf(x[t, e]):
                assert got[t, e] == 0
                continue
            up, down = x.copy(), x.copy()
            up[t, e] += 1e-6
            down[t, e] -= 1e-6
            assert abs((value(up) - value(down)) / 2e-6 - got[t, e]) < 1e-8
