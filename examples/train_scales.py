"""Training the activation factors of a frozen network against the next token: fake-quant in front of each frozen linear, the loss at a frozen output head.

    python examples/train_scales.py [--steps 40] [--per-channel]

Between forward and backward a step holds one byte for each input element of a linear (sasq_fakequant_fwd_ckpt) and nothing of the logits (sasq_linear_ce).
The factors start at what the largest activations ask for and are trained with AdamW; the whole step is one HIP graph.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_14481_amd import binding as B  # noqa: E402

BITS = 8


class Layer:
    """A frozen linear with the fake-quant operator in front of it: one factor, or one for each input channel."""

    def __init__(self, out_features: int, in_features: int, tokens: int, dtype: torch.dtype, per_channel: bool, g: torch.Generator):
        w = torch.randn(out_features, in_features, generator=g, device="cuda") * in_features ** -0.5
        wq = torch.empty(out_features, in_features, dtype=torch.int8, device="cuda")
        s_w = torch.empty(out_features, device="cuda")
        B.sasq_quantize_weight(w, wq, s_w)
        self.w = (wq.float() * s_w[:, None]).to(dtype)                  # what the frozen linear multiplies with while factors are trained
        self.wt = torch.empty(B.sasq_bwd_weight_bytes(out_features, in_features), dtype=torch.uint8, device="cuda")
        B.sasq_prepare_bwd_weight(wq, s_w, self.wt, out_features, in_features, B.SASQ_W_INT8, dtype)
        n = in_features if per_channel else 1
        self.s, self.ds = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
        self.m, self.v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        self.kept = torch.empty(tokens, in_features, dtype=torch.int8, device="cuda")
        self.xq = torch.empty(tokens, in_features, dtype=dtype, device="cuda")
        self.dx = torch.empty(tokens, in_features, dtype=dtype, device="cuda")
        need = B.sasq_fakequant_bwd_pc_ckpt_workspace if per_channel else B.sasq_fakequant_bwd_ckpt_workspace
        self.ws = B.new_workspace(max(need(tokens, in_features), B.sasq_absmax_scale_workspace(tokens, in_features)))
        self.fwd = B.sasq_fakequant_fwd_pc_ckpt if per_channel else B.sasq_fakequant_fwd_ckpt
        self.bwd = B.sasq_fakequant_bwd_pc_ckpt if per_channel else B.sasq_fakequant_bwd_ckpt

    def calibrate(self, x: torch.Tensor) -> None:
        s = torch.empty(1, device="cuda")
        B.sasq_absmax_scale(x, s, self.ws, BITS)
        self.s.copy_(s.expand_as(self.s))

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        self.fwd(x, self.s, self.xq, self.kept, BITS)
        return self.xq @ self.w.t()

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        """The gradient with respect to x; that of the factors goes to ds."""
        B.sasq_linear_bwd_input(dy, self.wt, self.dx, self.dx.shape[1])
        self.bwd(self.kept, self.dx, self.dx, self.ds, self.ws, BITS)
        return self.dx


class Network:
    """Linears one behind the other and an output head, all frozen; `step` is one pass of training but for the optimizer."""

    def __init__(self, tokens: int, hidden: int, inter: int, vocab: int, dtype: torch.dtype, per_channel: bool = False, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.layers = [Layer(inter, hidden, tokens, dtype, per_channel, g), Layer(hidden, inter, tokens, dtype, per_channel, g)]
        self.x = torch.randn(tokens, hidden, generator=g, device="cuda")
        self.x[:, ::50] *= 20                                           # outlier channels
        self.x = self.x.to(dtype)
        self.w = (torch.randn(vocab, hidden, generator=g, device="cuda") * hidden ** -0.5).to(dtype)
        self.heads = []
        for form in (B.SASQ_HEAD_LOGITS, B.SASQ_HEAD_GRAD):
            self.heads.append(torch.empty(B.sasq_head_bytes(vocab, hidden, form), dtype=torch.uint8, device="cuda"))
            B.sasq_prepare_head(self.w, self.heads[-1], form)
        h = self.x
        for layer in self.layers:                                       # factors from the activations that the network has without quantization
            layer.calibrate(h)
            h = h @ layer.w.t()
        self.targets = (h.float() @ self.w.float().t()).argmax(1).to(torch.int32)       # what it says without quantization
        self.targets[::7] = -100                                        # and tokens that are not trained on
        self.loss, self.mean = torch.empty(tokens, device="cuda"), torch.empty(1, device="cuda")
        self.dh = torch.empty(tokens, hidden, dtype=dtype, device="cuda")
        self.scale = 1024.0 if dtype == torch.float16 else 1.0          # gradients of a mean lie low in fp16
        self.ws = B.new_workspace(B.sasq_linear_ce_workspace(tokens, vocab, hidden, True))
        self.vocab = vocab

    def step(self) -> None:
        h = self.x
        for layer in self.layers:
            h = layer.forward(h)
        self.h = h
        B.sasq_linear_ce(h, self.heads[0], self.targets, self.loss, self.vocab, self.ws, mean=self.mean, dx=self.dh, head_grad=self.heads[1], scale=self.scale)
        d = self.dh
        for layer in reversed(self.layers):
            d = layer.backward(d)

    def update(self, number: int, lr: float) -> None:
        for layer in self.layers:
            B.sasq_scale_adamw(layer.s, layer.ds, layer.m, layer.v, number, lr, weight_decay=0.0)


def main(steps: int = 40, per_channel: bool = False, dtype: torch.dtype = torch.bfloat16) -> list[float]:
    net = Network(512, 512, 1408, 8000, dtype, per_channel)
    net.step()                                                          # everything loaded before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.step()
    losses = []
    for i in range(steps):
        graph.replay()
        net.update(i + 1, lr=2e-4)                                      # (AdamW: the gradient's scale does not matter)
        losses.append(net.mean.item())
        if i % 10 == 0 or i == steps - 1:
            print(f"step {i:3d}: loss {losses[-1]:.4f}", flush=True)
    return losses


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=40)
    p.add_argument("--per-channel", action="store_true")
    a = p.parse_args()
    main(a.steps, a.per_channel)
