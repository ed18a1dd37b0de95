"""The operators together, as a model uses them: tokens are embedded, a router chooses experts, these multiply, the results come back;
trained through autograd.Functions and served in 4 bits under a graph."""
import numpy as np
import pytest
import torch

import paper_2403_17017_amd as S
from oracle import routed_oracle as RO
from oracle import token_oracle as TO
from tests.gpu_util import announce
from tests.routed_util import U32, assert_within, host

pytestmark = pytest.mark.gpu
V, D, E, C, H, T = 60, 40, 16, 3, 24, 90


class Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, token, table, scale):
        ctx.save_for_backward(token)
        ctx.scale, ctx.rows = scale, table.shape[0]
        return S.seer_embed(token, table, scale=scale)

    @staticmethod
    def backward(ctx, dy):
        return None, S.seer_embed_grad(ctx.saved_tensors[0], dy.contiguous(), ctx.rows, scale=ctx.scale), None


class Choose(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, bias, how):
        expert, weight = S.seer_route_choose(logits, how, bias=bias)
        ctx.save_for_backward(logits, expert)
        ctx.how = how
        ctx.mark_non_differentiable(expert)
        return expert, weight

    @staticmethod
    def backward(ctx, _, dweight):
        logits, expert = ctx.saved_tensors
        return S.seer_route_choose_grad(logits, ctx.how, expert, dweight.contiguous()), None, None


class There(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, r):
        ctx.r = r
        return S.seer_route_gather(r, x)

    @staticmethod
    def backward(ctx, drows):
        return S.seer_route_combine(ctx.r, drows.contiguous()), None


class Back(torch.autograd.Function):
    @staticmethod
    def forward(ctx, z, weight, r):
        ctx.save_for_backward(z, weight)
        ctx.r = r
        return S.seer_route_combine(r, z, weight=weight)

    @staticmethod
    def backward(ctx, dy):
        z, weight = ctx.saved_tensors
        return (*S.seer_route_grad(ctx.r, dy.contiguous(), z, weight=weight), None)


def weights(seed, device="cuda:0"):
    g = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *s, by: torch.randn(*s, generator=g, device=device) * by
    return normal(V, D, by=0.3), normal(E, D, by=D ** -0.5), normal(E, H, D, by=D ** -0.5), normal(E, D, H, by=H ** -0.5)


@pytest.mark.parametrize("how", [dict(score="softmax"), dict(score="sigmoid", groups=4, best_groups=2, group_best=2, factor=2.5), dict(score="softmax", renormalise=False)], ids=str)
def test_gradients_of_a_model(how):
    announce(f"model {how}")
    how = {"choices": C, **how}
    leaves = [w.requires_grad_() for w in weights(1)]
    table, router, w1, w2 = leaves
    g = torch.Generator(device="cuda:0").manual_seed(2)
    token = torch.randint(-1, V, (T,), generator=g, device="cuda:0")
    bias = torch.randn(E, generator=g, device="cuda:0") * 0.05 if how["score"] == "sigmoid" else None
    c = torch.randn(T, D, generator=g, device="cuda:0")
    case = S.Choice(**how)

    def model():
        x = Embed.apply(token, table, 6.0)
        expert, weight = Choose.apply(x @ router.t(), bias, case)
        r = S.seer_route(expert, E)
        rows, ends = There.apply(x, r), r.expert_ptr.tolist()
        z = [torch.relu(rows[a:b] @ w1[e].t()) @ w2[e].t() for e, (a, b) in enumerate(zip(ends, ends[1:]))]
        return Back.apply(torch.cat(z + [torch.zeros_like(rows[ends[-1]:])]), weight, r) + x, expert
    y, expert = model()
    (y * c).sum().backward()
    # automatic differentiation of the formula in 64 bits, with the same experts
    t64, r64, a64, b64 = leaves64 = [w.detach().double().cpu().requires_grad_() for w in leaves]
    tok, e = token.cpu(), expert.cpu().long()
    x = torch.where((tok >= 0)[:, None], 6.0 * t64[tok.clamp(min=0)], torch.zeros((), dtype=torch.float64))
    logits = x @ r64.t()
    s = torch.softmax(logits, 1) if how["score"] == "softmax" else torch.sigmoid(logits)
    s = s.gather(1, e.clamp(min=0)) * (e >= 0)
    w = how.get("factor", 1.0) * (s / s.sum(1, keepdim=True) if how.get("renormalise", True) else s)
    want = x
    for k in range(C):
        hidden = torch.relu((a64[e[:, k]] @ x[:, :, None])[:, :, 0])
        want = want + w[:, k, None] * (b64[e[:, k]] @ hidden[:, :, None])[:, :, 0]
    want_e, _ = TO.choose(host(logits), C, bias=None if bias is None else host(bias), **{k: v for k, v in how.items() if k != "choices"})
    assert np.array_equal(host(expert), want_e)
    (want * c.double().cpu()).sum().backward()
    # chains of products and sums of at most some hundred fp32 terms: 2^-24 of their magnitudes each, which are within a factor of ten of the results
    near = lambda got, ref: float((got.double().cpu() - ref).norm()) <= 1e-4 * float(ref.norm())
    assert near(y.detach(), want.detach())
    assert all(near(a.grad, b.grad) for a, b in zip(leaves, leaves64))
    # once more, from the same leaves: the same bits
    first = [t.grad.clone() for t in leaves]
    for t in leaves:
        t.grad = None
    (model()[0] * c).sum().backward()
    assert torch.equal(first[0], table.grad) and torch.equal(first[1], router.grad)


def test_served_in_4_bits():
    """One layer of 4-bit products against their definition, and two layers captured and replayed."""
    announce("served in 4 bits")
    table, router, w1, w2 = weights(3)
    how = S.Choice(C, score="sigmoid", groups=4, best_groups=2, group_best=2)
    bits = [tuple(t.view(E, w.shape[1], -1) for t in S.seer_mx4_quantize(w.reshape(-1, w.shape[2]))) for w in (w1, w2)]
    token = torch.zeros(T, dtype=torch.int64, device="cuda:0")

    def serve(layers=2, stop=None):
        x = S.seer_embed(token, table, scale=6.0)
        expert, weight = S.seer_route_choose(x @ router.t(), how)
        r = S.seer_route(expert, E)
        q, scale = S.seer_route_gather_mx4(r, x)
        z = S.seer_mx4_product(q, scale, *bits[0], group_ptr=r.expert_ptr, dtype=torch.float32)
        if layers == 1:
            return x, expert, weight, S.seer_route_combine(r, z, weight=weight)
        z = S.seer_mx4_product(*S.seer_mx4_quantize(torch.relu(z)), *bits[1], group_ptr=r.expert_ptr, dtype=torch.float32)
        return S.seer_route_combine(r, z, weight=weight)
    g = torch.Generator(device="cuda:0").manual_seed(4)
    token.copy_(torch.randint(-1, V, (T,), generator=g, device="cuda:0"))
    x, expert, weight, y = serve(1)
    rows = RO.mx4_values(*RO.mx4_quantize(host(x)))
    w = RO.mx4_values(host(bits[0][0]), host(bits[0][1]))
    want, size = np.zeros((T, H)), np.zeros((T, H))
    for t in range(T):
        for k in range(C):
            e, p = host(expert)[t, k], host(weight)[t, k]
            want[t] += p * (w[e] @ rows[t])
            size[t] += p * (np.abs(w[e]) @ np.abs(rows[t]))
    assert_within(host(y), want, U32 * (C + 20) * size, "one layer")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            serve()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = serve()
    for _ in range(4):
        token.copy_(torch.randint(-1, V, (T,), generator=g, device="cuda:0"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, serve())


@pytest.mark.parametrize("op", ["choose", "embed", "mx4"])
def test_histories_are_refused(op):
    table, router, w1, _ = (w.requires_grad_() for w in weights(5))
    token = torch.zeros(4, dtype=torch.int64, device="cuda:0")
    call = {"choose": lambda: S.seer_route_choose(table, S.Choice(2)), "embed": lambda: S.seer_embed(token, table), "mx4": lambda: S.seer_mx4_quantize(table)}[op]
    with pytest.raises(RuntimeError, match="history"):
        call()
    with torch.no_grad():
        call()
