"""A layer of experts, trained and then used a token at a time, on the layer operators.

  python -m paper_1909_10616_amd.expert_layer [--tokens 4096] [--width 512] [--hidden 1024]
      [--experts 16] [--top 2] [--steps 200] [--dtype bf16] [--rate 3e-3] [--seed 0]

The model is Y = head(X + Σ_s w_s·expert_{e_s}(X)): a router product (gt_linear), the
choice of `top` experts a token (gt_route), their gated layers (gt_experts, the
residual fused) and a head (gt_linear). It learns synthetic data: tokens of
several kinds, each with a map of its own, so that the experts have something to
divide. A training step is the forward calls, their gradients
(gt_linear_backward, gt_experts_backward, gt_route_backward) and Adam on fp32
copies of the weights; a routing bias follows the experts' loads, which evens them
without a loss of its own. Afterwards single tokens run through the same
calls, captured once into a HIP graph, and must agree with the batch.
"""
from __future__ import annotations

import argparse
import time

from . import layers as L


class ExpertLayer:
    """The weights (fp32, and copies in the compute type) and the calls over them."""

    def __init__(self, width, hidden, experts, top, out, dtype, seed=0, device="cuda"):
        import torch
        gen = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, fan):
            return torch.randn(*shape, generator=gen, device=device) * fan ** -0.5

        self.top, self.dtype = top, dtype
        self.weights = {
            "router": normal(width, experts, fan=width),
            "W1": normal(experts, width, 2 * hidden, fan=width),
            "b1": torch.zeros(experts, 2 * hidden, device=device),
            "W2": normal(experts, hidden, width, fan=hidden),
            "b2": torch.zeros(experts, width, device=device),
            "head": normal(width, out, fan=width),
            "bias": torch.zeros(out, device=device),
        }
        self.first = {n: torch.zeros_like(w) for n, w in self.weights.items()}
        self.second = {n: torch.zeros_like(w) for n, w in self.weights.items()}
        self.steps = 0
        self.low = {n: w.to(dtype) for n, w in self.weights.items()}
        self.balance = torch.zeros(experts, device=device)

    def forward(self, X, keep=None, route=None):
        """Y; keep: a dict that receives what the gradients need. route: use this choice."""
        import torch
        w = self.low
        logits = L.gt_linear(X, w["router"])
        if route is None:
            route = L.gt_route(logits, self.top, bias=self.balance, score="softmax")
        P = None
        if keep is not None:
            P = torch.empty(X.shape[0] * self.top, w["W1"].shape[2], dtype=X.dtype, device=X.device)
        H = L.gt_experts(X, route, w["W1"], w["W2"], b1=w["b1"], b2=w["b2"], residual=X, act="silu",
                         gated=True, P=P)
        Y = L.gt_linear(H, w["head"], bias=w["bias"])
        if keep is not None:
            keep.update(X=X, logits=logits, route=route, P=P, H=H)
        return Y

    def backward(self, dY, kept):
        """The gradients of every weight, from the loss's with respect to Y."""
        w, X, route = self.low, kept["X"], kept["route"]
        dH, head, bias = L.gt_linear_backward(dY, kept["H"], w["head"], act="none")
        g = L.gt_experts_backward(dH, X, route, w["W1"], w["W2"], kept["P"], b2=w["b2"], act="silu",
                                  gated=True, need=("dW1", "dW2", "dweights"))
        dlogits = L.gt_route_backward(g.dweights, kept["logits"], route.experts, score="softmax")
        _, router, _ = L.gt_linear_backward(dlogits, X, w["router"], act="none", bias=False,
                                            need=("dW",))
        return {"router": router, "W1": g.dW1, "b1": g.db1, "W2": g.dW2, "b2": g.db2, "head": head,
                "bias": bias}

    def step(self, grads, route, rate, b1=0.9, b2=0.99, eps=1e-8):
        """Adam, then the routing bias a step towards even loads."""
        self.steps += 1
        for n, g in grads.items():
            g = g.float()
            self.first[n].lerp_(g, 1 - b1)
            self.second[n].lerp_(g * g, 1 - b2)
            m = self.first[n] / (1 - b1 ** self.steps)
            v = self.second[n] / (1 - b2 ** self.steps)
            self.weights[n].addcdiv_(m, v.sqrt().add_(eps), value=-rate)
            self.low[n].copy_(self.weights[n])
        load = route.offsets.diff().float()
        self.balance.add_((load.mean() - load).sign(), alpha=0.02)


class Task:
    """Tokens of `kinds` kinds: a kind's centre plus noise, and tanh of a map of its own."""

    def __init__(self, width, out, kinds, seed=1, device="cuda"):
        import torch
        self.gen = torch.Generator(device=device).manual_seed(seed)
        self.device = device
        self.centres = torch.randn(kinds, width, generator=self.gen, device=device)
        self.maps = torch.randn(kinds, width, out, generator=self.gen, device=device) * width ** -0.5

    def draw(self, tokens):
        import torch
        kind = torch.randint(len(self.centres), (tokens,), generator=self.gen, device=self.device)
        x = self.centres[kind]
        x = x + 0.5 * torch.randn(x.shape, generator=self.gen, device=self.device)
        y = torch.empty(tokens, self.maps.shape[2], device=self.device)
        for k, m in enumerate(self.maps):
            y[kind == k] = torch.tanh(x[kind == k] @ m)
        return x, y


def train(model, task, tokens, steps, rate, report=None):
    """The loss (mean square) of every step."""
    losses = []
    for i in range(steps):
        x, target = task.draw(tokens)
        kept = {}
        Y = model.forward(x.to(model.dtype), keep=kept)
        diff = Y.float() - target
        losses.append((diff * diff).mean())
        dY = (diff * (2.0 / diff.numel())).to(model.dtype)
        grads = model.backward(dY, kept)
        model.step(grads, kept["route"], rate)
        if report and (i % report == 0 or i == steps - 1):
            load = kept["route"].offsets.diff()
            print(f"step {i:4d}  loss {losses[-1].item():.4f}  rows of an expert "
                  f"{int(load.min())} … {int(load.max())}", flush=True)
    return [v.item() for v in losses]


class Server:
    """Single tokens: the forward calls captured once, replayed for every token."""

    def __init__(self, model, width):
        import torch
        self.x = torch.zeros(1, width, dtype=model.dtype, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            model.forward(self.x)
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.y = model.forward(self.x)

    def __call__(self, x):
        """The output of one token [1, width], valid until the next call."""
        self.x.copy_(x)
        self.graph.replay()
        return self.y


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 4096), ("width", 512), ("hidden", 1024), ("experts", 16), ("top", 2),
                        ("out", 256), ("kinds", 8), ("steps", 200), ("seed", 0), ("serve", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--rate", type=float, default=3e-3)
    ap.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    o = ap.parse_args(argv)
    dtype = torch.bfloat16 if o.dtype == "bf16" else torch.float32
    model = ExpertLayer(o.width, o.hidden, o.experts, o.top, o.out, dtype, o.seed)
    task = Task(o.width, o.out, o.kinds, o.seed + 1)
    begin = time.perf_counter()
    losses = train(model, task, o.tokens, o.steps, o.rate, report=max(1, o.steps // 10))
    torch.cuda.synchronize()
    took = time.perf_counter() - begin
    print(f"{o.steps} steps of {o.tokens} tokens: {1e3 * took / o.steps:.2f} ms a step "
          f"(data and optimiser included), loss {losses[0]:.4f} → {losses[-1]:.4f}")

    x, _ = task.draw(o.serve)
    x = x.to(dtype)
    batch = model.forward(x).float()
    server = Server(model, o.width)
    worst, begin = 0.0, time.perf_counter()
    single = [server(x[i:i + 1]).float().clone() for i in range(o.serve)]
    torch.cuda.synchronize()
    took = time.perf_counter() - begin
    worst = max(float((s[0] - batch[i]).abs().max()) for i, s in enumerate(single))
    print(f"{o.serve} single tokens: {1e6 * took / o.serve:.0f} µs each, largest difference from the batch "
          f"{worst:.1e} of {float(batch.abs().max()):.2f}")
    return losses, worst


if __name__ == "__main__":
    main()
