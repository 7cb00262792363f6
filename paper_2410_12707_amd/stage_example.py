"""A pipeline stage in training between two slow links: the feed-forward half of a transformer block.

    python -m paper_2410_12707_amd.stage_example

Activations come in and go out as compressed messages, gradients come back the same way (paper Sec. 3.3 and 5.1), and while several micro-batches
are under way (Sec. 3.6) each one's activations wait in 8 bits:

    forward    message -> x;  h, a = layer norm(x) (h kept);  z = a W1' + b1;  g = GELU(z) (z and g kept);  out = x + g W2' + b2 -> message
    backward   message -> dout;  dW2 += dout' g;  dg = dout W2;  dz = dg GELU'(z);  dW1 += dz' a;  da = dz W1;
               dx = layer norm's gradient + dout -> message

The matrix products between activations and weights are torch's; everything else is this package's.
"""
from __future__ import annotations

import torch

from . import binding as B

EPS = 1e-5


class FeedForwardStage:
    """Weights, their gradients, and what is kept of each micro-batch under way."""

    def __init__(self, features: int, hidden: int, tokens: int, micro_batches: int, dtype=torch.bfloat16, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(*shape, device="cuda", generator=gen) * scale).to(dtype)

        self.dtype, self.tokens, self.features, self.hidden = dtype, tokens, features, hidden
        self.weight = (1.0 + normal(features, scale=0.1).float()).to(dtype)
        self.bias = normal(features, scale=0.1)
        self.w1, self.b1 = normal(hidden, features, scale=features ** -0.5), normal(hidden, scale=0.1)
        self.w2, self.b2 = normal(features, hidden, scale=hidden ** -0.5), normal(features, scale=0.1)
        shapes = {"weight": (features,), "bias": (features,), "w1": (hidden, features), "b1": (hidden,), "w2": (features, hidden), "b2": (features,)}
        self.grad = {name: torch.zeros(*shape, device="cuda") for name, shape in shapes.items()}
        self.kept = [{"h": B.new_act8(tokens, features), "z": B.new_act8(tokens, hidden), "g": B.new_act8(tokens, hidden),
                      "rstd": torch.empty(tokens, device="cuda")} for _ in range(micro_batches)]
        need = max(B.adatopk_weight_grad_workspace_bytes(tokens, hidden, features, dtype), B.adatopk_weight_grad_workspace_bytes(tokens, features, hidden, dtype),
                   B.adatopk_layernorm_backward_workspace_bytes(tokens, features))
        self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")

    def kept_bytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in self.kept[0].values())

    def forward(self, x: torch.Tensor, m: int) -> torch.Tensor:
        kept, a = self.kept[m], torch.empty_like(x)
        B.adatopk_layernorm_forward(x, self.weight, self.bias, EPS, a, None, kept["rstd"], act8=kept["h"])
        z = torch.addmm(self.b1, a, self.w1.t())
        B.adatopk_gelu_forward(z, z, kept["z"], kept["g"], tanh=True)  # in place: z itself waits in 8 bits
        return torch.addmm(self.b2, z, self.w2.t()).add_(x)

    def backward(self, dout: torch.Tensor, m: int) -> torch.Tensor:
        kept, g = self.kept[m], self.grad
        B.adatopk_weight_grad(dout, kept["g"], g["w2"], g["b2"], self.workspace, accumulate=True)
        dz = torch.mm(dout, self.w2)
        B.adatopk_gelu_backward(dz, kept["z"], dz, tanh=True)
        B.adatopk_weight_grad(dz, kept["h"], g["w1"], g["b1"], self.workspace, weight=self.weight, bias=self.bias, accumulate=True)
        dx = torch.mm(dz, self.w1)
        B.adatopk_layernorm_backward(dx, None, kept["h"], None, kept["rstd"], self.weight, dx, g["weight"], g["bias"], self.workspace, dsum=dout, accumulate=True)
        return dx


class Link:
    """One direction of a slow link: a dense tensor as a message of its k largest values, and back."""

    def __init__(self, n: int, ratio: float, dtype=torch.bfloat16):
        code = B._dtype_code(dtype)
        self.ratio, self.k = ratio, B.adatopk_k_for_ratio(n, ratio)
        self.message = torch.empty(B.adatopk_wire_bytes(self.k, code, 4), dtype=torch.uint8, device="cuda")
        self.workspace = B.new_workspace(n, 1, dtype)

    def send(self, x: torch.Tensor) -> torch.Tensor:
        B.adatopk_compress_wire(x, self.k, 4, self.ratio, self.message, self.workspace)
        return self.message

    def receive(self, message: torch.Tensor, like: torch.Tensor) -> torch.Tensor:
        out = torch.empty_like(like)
        B.adatopk_decompress_wire(message, message.numel(), 4, out)
        return out


def train_step(stage: FeedForwardStage, inputs, gradients, link_in: Link, link_out: Link):
    """All forward passes, then all backward passes: the outgoing activations and gradients as the neighbours receive them."""
    for t in stage.grad.values():
        t.zero_()
    outs, dxs = [], []
    for m, x in enumerate(inputs):
        y = stage.forward(link_in.receive(link_in.send(x), x), m)
        outs.append(link_out.receive(link_out.send(y), y))
    for m, dout in enumerate(gradients):
        dx = stage.backward(link_out.receive(link_out.send(dout), dout), m)
        dxs.append(link_in.receive(link_in.send(dx), dx))
    return outs, dxs


def main(features: int = 1024, hidden: int = 4096, tokens: int = 2048, micro_batches: int = 4, ratio: float = 4.0) -> None:
    stage = FeedForwardStage(features, hidden, tokens, micro_batches)
    link_in, link_out = Link(tokens * features, ratio), Link(tokens * features, ratio)
    xs = [torch.randn(tokens, features, device="cuda").to(torch.bfloat16) for _ in range(micro_batches)]
    ds = [(torch.randn(tokens, features, device="cuda") * 1e-3).to(torch.bfloat16) for _ in range(micro_batches)]
    train_step(stage, xs, ds, link_in, link_out)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    train_step(stage, xs, ds, link_in, link_out)
    end.record()
    torch.cuda.synchronize()
    plain = 2 * tokens * (2 * features + 2 * hidden)  # x, a, z and g in 16 bits
    print("%d micro-batches of %d tokens, %d -> %d -> %d: %.2f ms a step; %.1f MB kept per micro-batch (%.1f MB in 16 bits); |dW1| = %.3e" % (
        micro_batches, tokens, features, hidden, features, begin.elapsed_time(end), stage.kept_bytes() / 1e6, plain / 1e6, float(stage.grad["w1"].norm())))


if __name__ == "__main__":
    main()
