"""seer_route_choose and seer_route_choose_grad against their definitions."""
import numpy as np
import pytest
import torch

import paper_2403_17017_amd as S
from oracle import token_oracle as O
from tests.gpu_util import announce
from tests.routed_util import ROUND, TINY, TYPES, U32, assert_within, host, rounded, shifted, spread

pytestmark = pytest.mark.gpu


def share_error(x, expert, choices, score, renormalise):
    """What a weight computed in fp32 may be off by, relative to itself [tokens, 1]: an exponential is off by 2 units in the last place
    and by its argument's rounding, half a unit of |x - top| (|x| of a sigmoid); one plus it, a quotient, a product and the
    factor add 8 units, a sum one for each of its terms."""
    E = x.shape[1]
    finite = np.where(np.isfinite(x), x, 0)
    span = finite.max(1, keepdims=True) - finite.min(1, keepdims=True) if score == "softmax" else np.abs(finite).max(1, keepdims=True)
    terms = choices if renormalise else E if score == "softmax" else 1
    return U32 * (24 + 2 * terms + 2 * span)


def check(x, kind, choices, rng, bias=None, grad=True, **how):
    """x float64 [T, E] of values that the type holds."""
    case = S.Choice(choices, **how)
    logits = rounded(x, kind)
    x = host(logits)
    b = None if bias is None else torch.from_numpy(np.asarray(bias, np.float32)).cuda()
    expert, weight = S.seer_route_choose(logits, case, bias=b)
    want_e, want_w = O.choose(x, choices, bias=None if bias is None else host(b), **how)
    assert expert.dtype == torch.int32 and np.array_equal(host(expert), want_e)
    err = share_error(x, want_e, choices, how.get("score", "softmax"), how.get("renormalise", True))
    got = host(weight)
    assert np.array_equal(np.isnan(got), np.isnan(want_w))
    ok = np.where(np.isnan(want_w), 0, want_w)
    assert_within(np.where(np.isnan(got), 0, got), ok, err * np.abs(ok) + 2.0 ** -126, "weight")
    if not grad:
        return
    dw = rng.standard_normal(want_w.shape).astype(np.float32)
    d = S.seer_route_choose_grad(logits, case, expert, torch.from_numpy(dw).cuda())
    check_grad(host(d), x, kind, want_e, dw, err, **how)


def check_grad(d, x, kind, expert, dw, err, **how):
    want, size = O.choose_grad(x, expert, dw.astype(np.float64), **{k: v for k, v in how.items() if k in ("score", "renormalise", "factor")})
    # a weight's error in each of two places, one more score, a sum over the choices and three products
    off = (3 * err + U32 * (8 + expert.shape[1])) * size + 2.0 ** -120
    assert_within(d, want, off + (np.abs(want) + off) * ROUND[kind] + TINY[kind], "dlogits")


SHAPES = [  # tokens, experts, choices, groups, best_groups, group_best
    (1, 1, 1, 1, 1, 1), (1, 256, 8, 8, 4, 2), (5, 8, 2, 1, 1, 1), (3, 8, 8, 1, 1, 1), (33, 160, 6, 8, 3, 1), (64, 64, 1, 1, 1, 1), (17, 65, 7, 1, 1, 1),
    (9, 72, 5, 9, 2, 2), (7, 12, 3, 4, 1, 2), (6, 16, 4, 16, 4, 1), (5, 16, 4, 16, 4, 2), (13, 300, 10, 3, 2, 2), (11, 512, 10, 8, 8, 2), (4, 1000, 16, 40, 7, 2),
    (3, 4096, 64, 64, 5, 2), (2, 4095, 64, 1, 1, 1), (130, 128, 8, 1, 1, 1), (21, 257, 9, 1, 1, 1), (6, 130, 64, 2, 2, 1), (8, 100, 20, 5, 3, 2), (10, 48, 3, 3, 1, 1),
    (1, 3, 2, 1, 1, 1), (4, 24, 6, 8, 3, 1), (29, 256, 8, 4, 2, 2), (67, 32, 4, 1, 1, 1),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("how", [("softmax", False, True), ("softmax", False, False), ("softmax", True, True), ("softmax", True, False), ("sigmoid", False, True),
                                 ("sigmoid", True, True), ("sigmoid", True, False)], ids=lambda h: f"{h[0]}{'+bias' if h[1] else ''}{'/sum' if h[2] else ''}")
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_choice(shape, how, kind):
    T, E, C, G, best, two = shape
    score, biased, renormalise = how
    announce(f"choose {shape} {how} {kind}")
    rng = np.random.default_rng(E * 7 + T)
    x = rng.standard_normal((T, E)) * 2
    bias = rng.standard_normal(E) * 0.1 if biased else None
    check(x, kind, C, rng, bias, score=score, groups=G, best_groups=best, group_best=two, renormalise=renormalise, factor=2.5 if renormalise else 1.0)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [None, 0.0])
@pytest.mark.parametrize("groups", [(1, 1, 1), (8, 2, 1), (8, 3, 2)], ids=str)
def test_ties_go_to_the_lower_number(groups, bias, score):
    """Three different logits among 96 experts, and rows that are all the same."""
    announce(f"ties {groups} {bias} {score}")
    rng = np.random.default_rng(5)
    x = rng.integers(0, 3, (40, 96)).astype(np.float64)
    x[3] = 1.0
    x[4] = -2.0
    G, best, two = groups
    check(x, "bf16", 9, rng, None if bias is None else np.zeros(96), score=score, groups=G, best_groups=best, group_best=two)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_masks(score, renormalise):
    """Experts out of service, rows with fewer than are wanted, rows with none, groups with none."""
    announce(f"masks {score} {renormalise}")
    rng = np.random.default_rng(6)
    x = rng.standard_normal((24, 64))
    x[:, 5] = -np.inf
    x[1] = -np.inf
    x[2, 3:] = -np.inf
    x[3, :63] = -np.inf
    x[4, :48] = -np.inf
    x[5, 16:] = -np.inf
    x[6, rng.random(64) < 0.9] = -np.inf
    bias = rng.standard_normal(64) * 0.1
    bias[7] = -np.inf
    for b in (None, bias):
        for G, best, two in ((1, 1, 1), (4, 2, 1), (4, 2, 2), (16, 3, 2), (64, 9, 2)):
            check(x, "f32", 6 if G < 64 else 9, rng, b, score=score, renormalise=renormalise, groups=G, best_groups=best, group_best=two)


def test_scores_that_32_bits_would_not_tell_apart():
    """Sigmoids of 17 and more are 1 in fp32, and a bias of 64 leaves a score 2^-17; in 64 bits they differ."""
    rng = np.random.default_rng(7)
    x = 17 + rng.permutation(96).reshape(2, 48) * 0.125
    check(x, "f32", 8, rng, np.zeros(48), score="sigmoid")
    x = rng.standard_normal((30, 48))
    check(x, "f32", 8, rng, np.full(48, 64.0), score="sigmoid")
    check(x, "f32", 8, rng, np.full(48, 64.0), score="softmax")
    check(x * 1e-4, "f32", 8, rng, np.zeros(48), score="sigmoid", groups=6, best_groups=3, group_best=2)
    check(x * 1e-4, "f32", 8, rng, None, score="softmax", groups=6, best_groups=3, group_best=2)
    check(x * 1e-6, "f32", 8, rng, (rng.integers(-3, 3, 48) * 2.0 ** -24), score="sigmoid")


def test_scores_too_small_for_32_bits():
    """Renormalised without loss; their gradients are those of a softmax over the chosen."""
    rng = np.random.default_rng(8)
    x = -150 + rng.standard_normal((10, 40)) * 3
    check(x, "f32", 5, rng, score="sigmoid")
    check(x, "f32", 5, rng, np.zeros(40), score="sigmoid")
    x[:, 3] = 90
    check(x, "f32", 5, rng, score="softmax", renormalise=False)
    check(x[:, 4:], "f32", 5, rng, score="softmax", groups=4, best_groups=2, group_best=2)
    check(np.full((3, 8), 3e38) * [1, -1, 0.5, 0.25, -0.5, 0.1, 0, 1], "f32", 3, rng, score="softmax", grad=False)
    check(np.full((3, 8), 3e38) * [1, -1, 0.5, 0.25, -0.5, 0.1, 0, 1], "f32", 3, rng, score="sigmoid", grad=False)


@pytest.mark.parametrize("bias", [None, 0.0])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_nan_and_infinity_show(score, bias):
    """A NaN is chosen first and makes the weights NaN; an infinity is chosen, and a softmax over it is NaN."""
    announce(f"nan {score} {bias}")
    rng = np.random.default_rng(9)
    x = rng.standard_normal((6, 20))
    x[1, 7] = np.nan
    x[2, [4, 9]] = np.nan
    x[3, 11] = np.inf
    x[4, 12], x[4, :4] = np.nan, -np.inf
    for renormalise in (True, False):
        expert, weight = S.seer_route_choose(rounded(x, "f32"), S.Choice(4, score=score, renormalise=renormalise), bias=None if bias is None else torch.zeros(20, device="cuda:0"))
        e, w = host(expert), host(weight)
        want, _ = O.choose(x[[0, 5]], 4, score=score, bias=None if bias is None else np.zeros(20), renormalise=renormalise)
        assert np.array_equal(e[[0, 5]], want) and np.isfinite(w[[0, 5]]).all()
        if score == "sigmoid" or bias is None:
            assert e[1, 0] == 7 and list(e[2, :2]) == [4, 9] and e[3, 0] == 11 and e[4, 0] == 12
        assert np.isnan(w[1, 0]) and np.isnan(w[2, :2]).all() and np.isnan(w[4, 0])
        if score == "softmax":
            assert np.isnan(w[3]).any()
        assert (e >= 0).all() and not np.isin(e[4], range(4)).any()


@pytest.mark.parametrize("kind", list(TYPES))
def test_strides_and_odd_addresses(kind):
    rng = np.random.default_rng(10)
    x = rounded(rng.standard_normal((37, 61)), kind)
    how = S.Choice(5, score="sigmoid", renormalise=True)
    e, w = S.seer_route_choose(x, how)
    dw = torch.from_numpy(rng.standard_normal((37, 5)).astype(np.float32)).cuda()
    d = S.seer_route_choose_grad(x, how, e, dw)
    for other in (spread(x, 77), shifted(x, 1), spread(shifted(x, 3), 64)):
        e2, w2 = S.seer_route_choose(other, how)
        assert torch.equal(e, e2) and torch.equal(w, w2)
        room = torch.full((37, 80), 55.0, dtype=x.dtype, device="cuda:0")
        d2 = S.seer_route_choose_grad(other, how, e, dw, dlogits=room[:, :61])
        assert torch.equal(d, d2) and bool((room[:, 61:] == 55).all())
    room = torch.full((37 * 5 + 2,), 55, dtype=torch.int32, device="cuda:0")
    S.seer_route_choose(x, how, expert=room[1:-1].view(37, 5))
    assert torch.equal(room[1:-1].view(37, 5), e) and room[0] == 55 and room[-1] == 55


def test_many_tokens():
    announce("70 001 tokens")
    g = torch.Generator(device="cuda:0").manual_seed(1)
    x = torch.randn(70001, 64, generator=g, device="cuda:0")
    e, w = S.seer_route_choose(x, S.Choice(4))
    top = torch.sort(x, dim=1, descending=True, stable=True)
    assert torch.equal(e.long(), top.indices[:, :4])
    want = torch.softmax(top.values[:, :4].double(), 1)
    assert bool(((w - want).abs() <= 64 * U32 * want).all())
    dw = torch.randn(70001, 4, generator=g, device="cuda:0")
    d = S.seer_route_choose_grad(x, S.Choice(4), e, dw)
    part = want * (dw - (want * dw).sum(1, keepdim=True))
    dense = torch.zeros_like(x, dtype=torch.float64).scatter_(1, e.long(), part)
    assert float((d - dense).abs().max()) <= 200 * U32 * float(dw.abs().max())


def test_nothing_to_choose_from():
    x = torch.empty(0, 16, device="cuda:0")
    e, w = S.seer_route_choose(x, S.Choice(3))
    assert e.shape == (0, 3) and w.shape == (0, 3)
    assert S.seer_route_choose_grad(x, S.Choice(3), e, w).shape == (0, 16)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("kind", list(TYPES))
def test_gradient_of_any_choice(kind, renormalise, score):
    """Experts that no logit would have chosen, the same one twice, nobody's, and ones that are not there."""
    announce(f"choose_grad {score} {renormalise} {kind}")
    rng = np.random.default_rng(11)
    for T, E, C in ((9, 7, 4), (5, 70, 6), (3, 300, 64), (2, 2000, 3)):
        logits = rounded(rng.standard_normal((T, E)) * 2, kind)
        logits[0, 3] = -np.inf
        expert = rng.integers(-1, E, (T, C))
        expert[0, :3] = [3, 1, 1]
        expert[1] = -1
        expert[2 % T, 0] = E + 5 if T > 2 else 1
        expert[T - 1, 1] = -(1 << 31)
        dw = rng.standard_normal((T, C)).astype(np.float32)
        dw[1] = np.nan                                   # of choices that are none
        d = S.seer_route_choose_grad(logits, S.Choice(min(C, E), score=score, renormalise=renormalise, factor=-1.5), torch.from_numpy(expert.astype(np.int32)).cuda(),
                                     torch.from_numpy(dw).cuda())
        x = host(logits)
        check_grad(host(d), x, kind, expert, dw, share_error(x, expert, C, score, renormalise), score=score, renormalise=renormalise, factor=-1.5)


@pytest.mark.parametrize("score,renormalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_gradient_by_differences(score, renormalise):
    """Central differences of the kernel's own weights with steps of 2^-6: (x / 2^6)^2 / 6 of third derivatives of at most 1, and
    weights' roundings of some 2^-21 over a step of 2^-5."""
    g = torch.Generator(device="cuda:0").manual_seed(2)
    x = torch.randn(8, 16, generator=g, device="cuda:0")
    how = S.Choice(16, score=score, renormalise=renormalise)          # all are chosen, so that no step changes the choice
    e, w = S.seer_route_choose(x, how)
    dw = torch.rand(8, 16, generator=g, device="cuda:0")
    d = S.seer_route_choose_grad(x, how, e, dw)

    def value(x):
        e2, w2 = S.seer_route_choose(x, how)
        by_expert = torch.zeros(8, 16, dtype=torch.float64, device="cuda:0").scatter_(1, e2.long(), w2.double())
        return (by_expert.gather(1, e.long()) * dw).sum(1)
    h = 2.0 ** -6
    for i in range(16):
        step = torch.zeros_like(x)
        step[:, i] = h
        slope = (value(x + step) - value(x - step)) / (2 * h)
        assert float((slope - d[:, i]).abs().max()) <= 16 * (h * h / 6 + 2.0 ** -21 / (2 * h))


def test_on_another_stream_and_captured():
    announce("choose captured")
    g = torch.Generator(device="cuda:0").manual_seed(3)
    x = torch.randn(300, 256, generator=g, device="cuda:0")
    bias = torch.randn(256, generator=g, device="cuda:0") * 0.1
    dw = torch.randn(300, 8, generator=g, device="cuda:0")
    how = S.Choice(8, score="sigmoid", groups=8, best_groups=4, group_best=2, factor=2.5)
    want = [*S.seer_route_choose(x, how, bias=bias)]
    want.append(S.seer_route_choose_grad(x, how, want[0], dw))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [*S.seer_route_choose(x, how, bias=bias, stream=side)]
    got.append(S.seer_route_choose_grad(x, how, got[0], dw, stream=side))
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    out = [torch.empty_like(t) for t in want]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        S.seer_route_choose(x, how, bias=bias, expert=out[0], weight=out[1])
        S.seer_route_choose_grad(x, how, out[0], dw, dlogits=out[2])
    for k in range(4):
        x.copy_(torch.randn(300, 256, generator=g, device="cuda:0"))
        for t in out:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        want = [*S.seer_route_choose(x, how, bias=bias)]
        want.append(S.seer_route_choose_grad(x, how, want[0], dw))
        assert all(torch.equal(a, b) for a, b in zip(want, out))


@pytest.mark.parametrize("how", [dict(score="sigmoid", groups=8, best_groups=4, group_best=2), dict(score="softmax", renormalise=False), dict(score="softmax", groups=4, best_groups=2)], ids=str)
@pytest.mark.parametrize("E", [64, 256, 512])
def test_many_tokens_choose_as_64_bits_do(E, how):
    """40 000 tokens: experts equal to those of the definition, borders that 32 bits leave open among them."""
    announce(f"40 000 tokens of {E} {how}")
    g = torch.Generator(device="cuda:0").manual_seed(E)
    x = torch.randn(40000, E, generator=g, device="cuda:0") * 1.5
    bias = torch.round(torch.randn(E, generator=g, device="cuda:0") * 20) * 1e-3 if how["score"] == "sigmoid" else None
    e, _ = S.seer_route_choose(x, S.Choice(8, **how), bias=bias)
    d = x.double()
    s = torch.sigmoid(d) if how["score"] == "sigmoid" else torch.softmax(d, 1)
    key = d if bias is None else s + bias.double()
    if how.get("groups", 1) > 1:
        G = how["groups"]
        top = torch.sort(key.view(-1, G, E // G), dim=2, descending=True).values
        worth = top[:, :, :2].sum(2) if how.get("group_best") == 2 else top[:, :, 0]
        best = torch.sort(worth, dim=1, descending=True, stable=True).indices[:, : how["best_groups"]]
        shut = torch.ones(40000, G, dtype=torch.bool, device="cuda:0").scatter_(1, best, False)
        key = key.masked_fill(shut.repeat_interleave(E // G, 1), -float("inf"))
    want = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :8]
    assert torch.equal(e.long(), want)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [(1, 1, 1), (4, 2, 1), (4, 2, 2)], ids=str)
@pytest.mark.parametrize("E", [16, 64, 384])
def test_biases_at_the_ends_of_the_range(E, groups, score):
    """The lowest number as a mask, and sums and distances of two biases that 32 bits do not hold."""
    announce(f"choose biases {E} {groups} {score}")
    rng = np.random.default_rng(E)
    far = float(np.finfo(np.float32).max)
    x = rng.standard_normal((9, E)) * 2
    masked = np.where(rng.random(E) < 0.6, -far, rng.standard_normal(E) * 0.1)
    high = np.where(rng.random(E) < 0.3, far, 0.9 * far)
    both = rng.choice([-far, -0.75 * far, 0.0, 0.75 * far, far], E)
    one = np.full(E, -far)
    one[E // 3] = far
    two = rng.standard_normal(E) * 0.1
    two[[1, 2, E // 2, E // 2 + 1, E - 1, E - 2]] = [0.6 * far, 0.6 * far, 0.8 * far, 0.8 * far, 0.9 * far, 0.9 * far]
    for bias in (masked, high, both, one, two, -high):
        G, best, of = groups
        check(x, "f32", 4, rng, bias.astype(np.float32), grad=False, score=score, groups=G, best_groups=best, group_best=of)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [(2, 1, 1), (4, 2, 1), (4, 3, 1), (4, 2, 2)], ids=str)
@pytest.mark.parametrize("E", [16, 64, 384, 600])
def test_lowest_logits_beside_groups_with_none(E, groups, score):
    """Experts held back by fp32's lowest number are there, those with minus infinity are not: a group of the first kind comes before one of the second."""
    announce(f"choose lowest {E} {groups} {score}")
    rng = np.random.default_rng(E)
    G, best, of = groups
    n, lowest = E // G, float(np.finfo(np.float32).min)
    x = rng.standard_normal((2 * G + 2, E))
    for g in range(G):
        x[g, :] = lowest
        x[g, g * n: (g + 1) * n] = -np.inf                       # one group has none
        x[G + g, :] = -np.inf
        x[G + g, g * n: (g + 1) * n] = lowest                    # all but one have none
    x[2 * G, :n] = -np.inf
    x[2 * G, n:] = np.where(np.arange(E - n) % 3, lowest, -np.inf)
    x[2 * G + 1] = lowest
    for bias in (None, np.zeros(E)):
        check(x, "f32", min(3, n), rng, bias, grad=False, score=score, groups=G, best_groups=best, group_best=of)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("E", [8, 64, 300, 600])
def test_gradient_of_masked_logits_is_zero(E, kind, renormalise, score):
    """Whatever the others' gradients are: NaN, infinite, or of a row with a NaN in it."""
    announce(f"choose_grad masked {E} {kind} {renormalise} {score}")
    rng = np.random.default_rng(E)
    x = rng.standard_normal((7, E))
    masked = rng.random((7, E)) < 0.4
    masked[:, :3], masked[:, 3] = False, True
    x[masked] = -np.inf
    x[1, 0], x[2, 1] = np.nan, np.inf
    expert = np.tile([0, 1, 3], (7, 1)).astype(np.int32)
    dw = rng.standard_normal((7, 3)).astype(np.float32)
    dw[3, 0], dw[4, 1], dw[5, 0] = np.inf, np.nan, -np.inf
    d = host(S.seer_route_choose_grad(rounded(x, kind), S.Choice(3, score=score, renormalise=renormalise), torch.from_numpy(expert).cuda(), torch.from_numpy(dw).cuda()))
    assert not d[masked].any() and np.isfinite(d[[0, 6]]).all() and np.isnan(d[1]).any()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,C", [(8, 2), (64, 8), (256, 8), (300, 15), (512, 10), (600, 8), (64, 20)], ids=str)
@pytest.mark.parametrize("biased", [False, True])
def test_weights_are_rounded_once(E, C, biased, score):
    """Weights are computed in 64 bits and rounded to fp32: half a unit in the last place, and 2^-40 for the 64 bits."""
    announce(f"weights {E} {C} {score} {biased}")
    rng = np.random.default_rng(E + C)
    x = rounded(rng.standard_normal((200, E)) * 3, "f32")
    x[1] -= 150
    x[2] *= 10
    bias = (rng.standard_normal(E) * 0.1).astype(np.float32) if biased else None
    for renormalise in (True, False) if score == "sigmoid" else (True,):
        e, w = S.seer_route_choose(x, S.Choice(C, score=score, renormalise=renormalise, factor=2.5), bias=None if bias is None else torch.from_numpy(bias).cuda())
        want_e, want = O.choose(host(x), C, bias=None if bias is None else bias.astype(np.float64), score=score, renormalise=renormalise, factor=2.5)
        assert np.array_equal(host(e), want_e)
        assert_within(host(w), want, np.abs(want) * (U32 + 2.0 ** -40) + TINY["f32"], "weight")


@pytest.mark.parametrize("E", [8, 64, 160, 256, 300, 512])
def test_weights_of_a_softmax_over_all_experts(E):
    """The sum that they are divided by has terms in 32 bits: an exponential is off by 2 half units in the last place and by 2.25 of them for
    each unit of its argument (a difference, a product, and log2(e) in 32 bits), the sum by these on its terms' average and by 5 for up to 32
    terms added by halves; everything else is in 64 bits, and rounded once."""
    announce(f"weights of a softmax over {E}")
    rng = np.random.default_rng(E)
    x = host(rounded(rng.standard_normal((300, E)) * 3, "f32"))
    x[1] *= 8
    e, w = S.seer_route_choose(torch.from_numpy(x).float().cuda(), S.Choice(min(E, 8), renormalise=False))
    want_e, want = O.choose(x, min(E, 8), renormalise=False)
    assert np.array_equal(host(e), want_e)
    d = x.max(1, keepdims=True) - x
    terms = 5 + (np.exp(-d) * (2 + 2.25 * d)).sum(1, keepdims=True) / np.exp(-d).sum(1, keepdims=True)
    assert_within(host(w), want, want * (U32 * (1 + terms) * (1 + 2.0 ** -10)) + 2.0 ** -126, "weight")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("E", [1, 8, 64, 256, 512, 600])
def test_one_choice_renormalised_is_the_factor(E, kind, score):
    """Its weight hangs on no logit, so its gradient is 0."""
    announce(f"one choice of {E} {kind} {score}")
    rng = np.random.default_rng(E)
    x = rounded(rng.standard_normal((500, E)) * 4, kind)
    how = S.Choice(1, score=score, factor=2.7)
    e, w = S.seer_route_choose(x, how)
    assert bool((w == float(np.float32(2.7))).all())
    assert not S.seer_route_choose_grad(x, how, e, torch.from_numpy(rng.standard_normal((500, 1)).astype(np.float32)).cuda()).any()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [(2, 1, 2), (4, 3, 1), (8, 4, 2), (16, 5, 2)], ids=str)
@pytest.mark.parametrize("E", [16, 64, 256, 384])
def test_groups_with_none_beside_sums_of_any_size(E, groups, score):
    """Padding, fewer groups in service than are kept, one more, and groups whose two best have a sum below all numbers in 32 bits."""
    announce(f"choose padding {E} {groups} {score}")
    rng = np.random.default_rng(E)
    G, best, of = groups
    n, far = E // G, float(np.finfo(np.float32).max)
    x = rng.standard_normal((60, E)) * 2
    x[rng.random(60) < 0.2] = -np.inf
    for t in range(20):                                          # t + 1 groups of the row are in service
        keep = rng.permutation(G)[: t % G + 1]
        x[t] = np.where(np.isin(np.arange(E) // n, keep), x[t], -np.inf)
    low = -far * rng.choice([0.4, 0.7, 0.9, 1.0], E)
    some = np.where(rng.random(E) < 0.5, low, rng.standard_normal(E) * 0.1)
    for bias in (rng.standard_normal(E) * 0.1, low, some, np.zeros(E)) + ((None,) if of == 2 else ()):
        check(x, "f32", min(4, n), rng, None if bias is None else bias.astype(np.float32), grad=False, score=score, groups=G, best_groups=best, group_best=of)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("how", [dict(score="sigmoid"), dict(score="softmax", renormalise=False, bias=True), dict(score="sigmoid", groups=4, best_groups=2, group_best=2, bias=True),
                                 dict(score="softmax", groups=8, best_groups=3)], ids=str)
@pytest.mark.parametrize("E", [64, 192, 256, 512])
def test_strides_and_odd_addresses_of_four_at_a_time(E, how, kind):
    """Numbers of experts that rows are read four elements at a time for, at every address that an element can have."""
    announce(f"choose strides {E} {how} {kind}")
    rng = np.random.default_rng(E)
    how = dict(how)
    bias = torch.from_numpy((rng.standard_normal(E) * 0.1).astype(np.float32)).cuda() if how.pop("bias", False) else None
    case = S.Choice(5, **how)
    x = rounded(rng.standard_normal((37, E)), kind)
    e, w = S.seer_route_choose(x, case, bias=bias)
    want, _ = O.choose(host(x), 5, bias=None if bias is None else host(bias), **how)
    assert np.array_equal(host(e), want)
    dw = torch.from_numpy(rng.standard_normal((37, 5)).astype(np.float32)).cuda()
    d = S.seer_route_choose_grad(x, case, e, dw)
    for ld in (E, E + 1, E + 13):
        for by in (0, 1, 2, 3):
            room = torch.full((37 * ld + by,), float("nan"), dtype=x.dtype, device="cuda:0")
            other = room[by:].view(37, ld)[:, :E]
            other.copy_(x)
            e2, w2 = S.seer_route_choose(other, case, bias=bias)
            assert torch.equal(e, e2) and torch.equal(w, w2)
            to = torch.full((37 * ld + by,), 55.0, dtype=x.dtype, device="cuda:0")
            to_rows = to[by:].view(37, ld)
            assert torch.equal(S.seer_route_choose_grad(other, case, e, dw, dlogits=to_rows[:, :E]), d)
            assert bool((to_rows[:, E:] == 55).all()) and bool((to[:by] == 55).all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("score,renormalise", [("softmax", True), ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("E,C", [(8, 2), (64, 8), (256, 8), (300, 15), (512, 16), (600, 8), (64, 20)], ids=str)
def test_gradients_are_rounded_to_fp32_once(E, C, score, renormalise, kind):
    """Computed in 64 bits (2^-40 of the magnitudes that cancel), taken to fp32 and to the type."""
    announce(f"choose_grad rounding {E} {C} {score} {renormalise} {kind}")
    rng = np.random.default_rng(E + C)
    logits = rounded(rng.standard_normal((200, E)) * 3, kind)
    logits[1] -= 150
    x = host(logits)
    expert = np.stack([rng.permutation(E)[:C] for _ in range(200)]).astype(np.int32)
    dw = rng.standard_normal((200, C)).astype(np.float32)
    d = S.seer_route_choose_grad(logits, S.Choice(C, score=score, renormalise=renormalise, factor=2.5), torch.from_numpy(expert).cuda(), torch.from_numpy(dw).cuda())
    want, size = O.choose_grad(x, expert, dw.astype(np.float64), score=score, renormalise=renormalise, factor=2.5)
    off = np.abs(want) * U32 + size * 2.0 ** -40 + TINY["f32"]
    assert_within(host(d), want, off if kind == "f32" else off + (np.abs(want) + off) * ROUND[kind] + TINY[kind], "dlogits")
