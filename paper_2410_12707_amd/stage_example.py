"""A pipeline stage in training between two slow links: the feed-forward half of a transformer block.

    python -m paper_2410_12707_amd.stage_example [--eight-bit]

Activations come in and go out as compressed messages, gradients come back the same way (paper Sec. 3.3 and 5.1), and while several micro-batches
are under way (Sec. 3.6) each one's activations wait in 8 bits:

    forward    message -> x;  h, a = layer norm(x) (h kept);  z = a W1' + b1;  g = GELU(z) (z and g kept);  out = x + g W2' + b2 -> message
    backward   message -> dout;  dW2 += dout' g;  dg = dout W2;  dz = dg GELU'(z);  dW1 += dz' a;  da = dz W1;
               dx = layer norm's gradient + dout -> message

The matrix products between activations and weights are torch's; everything else is this package's.

With --eight-bit the norm is a root-mean-square norm and the projections, forward and backward, run in 8-bit floating point, from what the norm, GELU and the links
hand over; behind the last micro-batch the projections' weights are updated by their orthogonalised gradients and put into 8 bits again (the norm's weight and the biases, whose
gradients are there too, are a caller's to update).  Every product is this package's then.  It shows the calls together and is not faster at these sizes: GELU, its
backward pass and the links hand over dense rows, which four more launches per micro-batch put into 8 bits.
"""
from __future__ import annotations

import argparse

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


class EightBitStage(FeedForwardStage):
    """The same with projections in 8-bit floating point, a root-mean-square norm before them and updates of their weights."""

    def __init__(self, features: int, hidden: int, tokens: int, micro_batches: int, dtype=torch.bfloat16, seed: int = 0):
        super().__init__(features, hidden, tokens, micro_batches, dtype, seed)
        self.eight = {name: (B.new_fp8(*getattr(self, name).shape), B.new_fp8(*reversed(getattr(self, name).shape))) for name in ("w1", "w2")}
        self.momentum = {name: torch.zeros_like(self.grad[name]) for name in self.eight}
        need = max(B.adatopk_rmsnorm_backward_workspace_bytes(tokens, features), B.adatopk_muon_update_workspace_bytes(hidden, features),
                   B.adatopk_fp8_product_workspace_bytes(tokens, hidden, features), B.adatopk_fp8_product_workspace_bytes(tokens, features, hidden))
        if need > self.workspace.numel():
            self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        # what goes into a product and is done with behind it
        self.narrow, self.wide = B.new_fp8(tokens, features), B.new_fp8(tokens, hidden)
        self.put_away()

    def put_away(self) -> None:
        for name, (straight, across) in self.eight.items():
            B.adatopk_fp8_store_weight(getattr(self, name), straight, across)

    def forward(self, x: torch.Tensor, m: int) -> torch.Tensor:
        kept, z, out = self.kept[m], torch.empty(self.tokens, self.hidden, dtype=self.dtype, device="cuda"), torch.empty_like(x)
        B.adatopk_rmsnorm_forward(x, self.weight, EPS, None, kept["rstd"], act8=kept["h"], fp8=self.narrow)  # the weighted rows are wanted in 8 bits alone
        B.adatopk_fp8_product(self.narrow, self.eight["w1"][0], self.features, z, self.workspace, bias=self.b1)
        B.adatopk_gelu_forward(z, z, kept["z"], kept["g"], tanh=True)
        B.adatopk_fp8_store(z, self.wide)
        B.adatopk_fp8_product(self.wide, self.eight["w2"][0], self.hidden, out, self.workspace, bias=self.b2, add=x)
        return out

    def backward(self, dout: torch.Tensor, m: int) -> torch.Tensor:
        kept, g, dz, dx = self.kept[m], self.grad, torch.empty(self.tokens, self.hidden, dtype=self.dtype, device="cuda"), torch.empty_like(dout)
        B.adatopk_weight_grad(dout, kept["g"], g["w2"], g["b2"], self.workspace, accumulate=True)
        B.adatopk_fp8_store(dout, self.narrow)
        B.adatopk_fp8_product(self.narrow, self.eight["w2"][1], self.features, dz, self.workspace)
        B.adatopk_gelu_backward(dz, kept["z"], dz, tanh=True)
        B.adatopk_weight_grad(dz, kept["h"], g["w1"], g["b1"], self.workspace, weight=self.weight, accumulate=True)
        B.adatopk_fp8_store(dz, self.wide)
        B.adatopk_fp8_product(self.wide, self.eight["w1"][1], self.hidden, dx, self.workspace)
        B.adatopk_rmsnorm_backward(dx, None, kept["h"], kept["rstd"], self.weight, dx, g["weight"], self.workspace, dsum=dout, accumulate=True)
        return dx

    def update(self, rate: float = 0.02, decay: float = 0.1, mu: float = 0.95) -> None:
        """The projections' weights after a step's last micro-batch.  Coarse: their gradients come out of products in 8 bits, some percent off."""
        for name in self.eight:
            B.adatopk_muon_update(self.grad[name], self.momentum[name], mu, True, getattr(self, name), -rate, 1.0 - rate * decay, self.workspace, coarse=True)
        self.put_away()


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


def main(features: int = 1024, hidden: int = 4096, tokens: int = 2048, micro_batches: int = 4, ratio: float = 4.0, eight_bit: bool = False) -> None:
    stage = (EightBitStage if eight_bit else FeedForwardStage)(features, hidden, tokens, micro_batches)
    link_in, link_out = Link(tokens * features, ratio), Link(tokens * features, ratio)
    xs = [torch.randn(tokens, features, device="cuda").to(torch.bfloat16) for _ in range(micro_batches)]
    ds = [(torch.randn(tokens, features, device="cuda") * 1e-3).to(torch.bfloat16) for _ in range(micro_batches)]

    def step():
        train_step(stage, xs, ds, link_in, link_out)
        if eight_bit:
            stage.update()

    step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    step()
    end.record()
    torch.cuda.synchronize()
    plain = 2 * tokens * (2 * features + 2 * hidden)  # x, a, z and g in 16 bits
    print("%d micro-batches of %d tokens, %d -> %d -> %d%s: %.2f ms a step; %.1f MB kept per micro-batch (%.1f MB in 16 bits); |dW1| = %.3e" % (
        micro_batches, tokens, features, hidden, features, " in 8 bits" if eight_bit else "", begin.elapsed_time(end), stage.kept_bytes() / 1e6, plain / 1e6,
        float(stage.grad["w1"].norm())))


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description="A pipeline stage's training step between two compressed links.")
    parser.add_argument("--eight-bit", action="store_true", help="projections in 8-bit floating point, their weights updated")
    main(eight_bit=parser.parse_args().eight_bit)
