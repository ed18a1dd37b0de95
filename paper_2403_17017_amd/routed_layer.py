"""A small routed layer, trained and served with the library's operators (an example, and a check that they fit together):

    python -m paper_2403_17017_amd.routed_layer

Every token goes to `choices` of `experts` two-layer networks, y = sum_k p_k W2_e(k) relu(W1_e(k) x), with the router's softmax
over the chosen experts as weights.  Training: seer_route, seer_route_gather, seer_route_combine, their gradients by
seer_route_grad and seer_route_combine, and seer_grad_clip before the step; the experts' own products, which training does in
floating point, are torch's.  Serving: the same layer with 8-bit weights, seer_route_gather_i8, seer_i8_product,
seer_i8_quantize and seer_route_combine, with nothing coming back to the host.
"""
from __future__ import annotations

import argparse

import paper_2403_17017_amd as S


class RoutedLayer:
    def __init__(self, experts=8, choices=2, columns=64, hidden=128, seed=0, device="cuda:0"):
        import torch
        g = torch.Generator(device=device).manual_seed(seed)
        normal = lambda *shape, scale: torch.randn(*shape, generator=g, device=device) * scale
        self.experts, self.choices = experts, choices
        self.router = normal(experts, columns, scale=columns ** -0.5)
        self.w1 = normal(experts, hidden, columns, scale=columns ** -0.5)
        self.w2 = normal(experts, columns, hidden, scale=hidden ** -0.5)
        # where the gradients lie does not change from step to step, so their list is made once
        self.weights = [self.router, *self.w1, *self.w2]
        self.grads = [torch.zeros_like(w) for w in self.weights]
        self.tensors = S.GradTensors(self.grads)

    def choose(self, x):
        """(weights of the chosen experts, the experts) of every token."""
        import torch
        top, expert = torch.topk(x @ self.router.t(), self.choices, dim=1)
        return torch.softmax(top, dim=1), expert

    def forward(self, x):
        """(y, what backward needs)."""
        import torch
        weight, expert = self.choose(x)
        r = S.seer_route(expert, self.experts)
        rows = S.seer_route_gather(r, x)
        ends = r.expert_ptr.tolist()
        hidden, z = torch.zeros(rows.shape[0], self.w1.shape[1], device=x.device), torch.zeros_like(rows)
        for e in range(self.experts):
            mine = slice(ends[e], ends[e + 1])
            hidden[mine] = torch.relu(rows[mine] @ self.w1[e].t())
            z[mine] = hidden[mine] @ self.w2[e].t()
        return S.seer_route_combine(r, z, weight=weight), (x, weight, expert, r, rows, ends, hidden, z)

    def backward(self, dy, kept):
        """Fills self.grads; the gradient in x is returned."""
        import torch
        x, weight, expert, r, rows, ends, hidden, z = kept
        dz, dweight = S.seer_route_grad(r, dy, z, weight=weight)
        drows = torch.zeros_like(rows)
        E = self.experts
        for e in range(E):
            mine = slice(ends[e], ends[e + 1])
            dhidden = (dz[mine] @ self.w2[e]) * (hidden[mine] > 0)
            torch.mm(dz[mine].t(), hidden[mine], out=self.grads[1 + E + e])
            torch.mm(dhidden.t(), rows[mine], out=self.grads[1 + e])
            drows[mine] = dhidden @ self.w1[e]
        dx = S.seer_route_combine(r, drows)
        dtop = weight * (dweight - (weight * dweight).sum(1, keepdim=True))       # the softmax over the chosen
        dlogits = torch.zeros(x.shape[0], E, device=x.device).scatter_(1, expert, dtop)
        torch.mm(dlogits.t(), x, out=self.grads[0])
        return dx + dlogits @ self.router

    def step(self, x, target, rate=0.05, max_norm=1.0):
        """One step of gradient descent on the mean squared error: (loss, norm of the gradients before clipping)."""
        y, kept = self.forward(x)
        off = y - target
        self.backward(off * (2.0 / off.numel()), kept)
        norm = S.seer_grad_clip(self.tensors, max_norm)
        for w, g in zip(self.weights, self.grads):
            w -= rate * g
        return off.square().mean(), norm

    def serve(self, x):
        """The layer in 8-bit integers; asynchronous throughout."""
        import torch
        weight, expert = self.choose(x)
        r = S.seer_route(expert, self.experts)
        q, scale = S.seer_route_gather_i8(r, x)
        hidden = S.seer_i8_product(q, scale, *self.quantized[0], group_ptr=r.expert_ptr, dtype=torch.float32)
        q, scale = S.seer_i8_quantize(torch.relu_(hidden))
        z = S.seer_i8_product(q, scale, *self.quantized[1], group_ptr=r.expert_ptr, dtype=torch.float32)
        return S.seer_route_combine(r, z, weight=weight)

    def quantize(self):
        """Lays the weights out for serving: 8-bit integers, a scale for each channel."""
        self.quantized = []
        for w in (self.w1, self.w2):
            q, scale = S.seer_i8_quantize(w.reshape(-1, w.shape[2]))
            self.quantized.append((q.unflatten(0, w.shape[:2]), scale.view(w.shape[:2])))


def main(argv=None):
    import torch
    p = argparse.ArgumentParser(description="Trains a small routed layer and serves it in 8-bit integers.")
    p.add_argument("--tokens", type=int, default=4096)
    p.add_argument("--steps", type=int, default=200)
    a = p.parse_args(argv)
    teacher, layer = RoutedLayer(seed=1), RoutedLayer(seed=2)
    g = torch.Generator(device="cuda:0").manual_seed(3)
    x = torch.randn(a.tokens, 64, generator=g, device="cuda:0")
    target = teacher.forward(x)[0]
    losses = []
    for i in range(a.steps):
        loss, norm = layer.step(x, target, rate=2.0)
        if i % 20 == 0 or i == a.steps - 1:
            losses.append(float(loss))
            print(f"step {i}: loss {losses[-1]:.5f}, norm of the gradients {float(norm):.4f}", flush=True)
    layer.quantize()
    y, served = layer.forward(x)[0], layer.serve(x)
    off = float((served - y).norm() / y.norm())
    print(f"served in 8-bit integers: {off:.4f} off the same layer in 32 bits")
    return losses, off


if __name__ == "__main__":
    main()
