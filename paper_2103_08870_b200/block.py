"""A residual block trained on K nodes through the compressed gradient path: the layer operators and the compression
together, as a training program uses them.

    y = x + W2 leaky(W1 norm(x))

The nodes' tokens are K runs of rows of x.  What the backward pass needs is kept in 8 bits (x, norm(x), and the hidden
layer, whose sign is also the leaky ReLU's derivative); the products run on 8-bit operands; the gradients of gamma, beta,
W1 and W2 land per node in the rows of `grads`, which the compression context reads::

    python -m paper_2103_08870_b200.block --nodes 4 --rows 4096 --width 1024 --hidden 4096 --steps 40
"""
from __future__ import annotations

import argparse
from typing import Optional

import torch

from . import layers, lgc

SLOPE = 0.01
EPS = 1e-5


class ResidualBlock:
    """Parameters, 8-bit weights and the buffers of one step; parameters lie flat in the order gamma, beta, W1, W2."""

    def __init__(self, rows: int, width: int, hidden: int, num_nodes: int, device: Optional[torch.device] = None, seed: int = 0):
        if width % 8 or hidden % 8:
            raise ValueError("width and hidden: multiples of 8 (rows of the activations start 16-byte aligned)")
        dev = torch.device(device if device is not None else "cuda:0")
        torch.cuda.set_device(dev)                                        # (the calls run on the current device)
        self.rows, self.width, self.hidden, self.K = rows, width, hidden, num_nodes
        self.numel = [width, width, hidden * width, width * hidden]       # the layer table of the compression context
        at = [0]
        for n in self.numel:
            at.append(at[-1] + n)
        self.N, self.at = at[-1], at
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        self.theta = torch.zeros(self.N, device=dev)
        self.gamma, self.beta, w1, w2 = (self.theta[a:b] for a, b in zip(at[:-1], at[1:]))
        self.w1, self.w2 = w1.view(hidden, width), w2.view(width, hidden)
        self.gamma.fill_(1.0)
        self.w1.uniform_(-1, 1, generator=g).mul_(width ** -0.5)
        self.w2.uniform_(-1, 1, generator=g).mul_(hidden ** -0.5)
        self.w1_8, self.w2_8 = layers.packed_empty(hidden, width, 128, dev), layers.packed_empty(width, hidden, 128, dev)
        self.grads = torch.zeros(num_nodes, self.N, device=dev)
        bf = dict(dtype=torch.bfloat16, device=dev)
        self.mean, self.rstd = torch.empty(rows, device=dev), torch.empty(rows, device=dev)
        self.x8, self.h8, self.a8 = (layers.packed_empty(rows, n, device=dev) for n in (width, width, hidden))
        self.dy8, self.dz8 = layers.packed_empty(rows, width, device=dev), layers.packed_empty(rows, hidden, device=dev)
        self.y, self.dh, self.dx = (torch.empty(rows, width, **bf) for _ in range(3))
        self.da, self.dz = torch.empty(rows, hidden, **bf), torch.empty(rows, hidden, **bf)
        self.refresh()

    def refresh(self) -> None:
        """Rounds the weights to 8 bits; after every update of `theta`."""
        layers.pack(self.w1, self.w1_8)
        layers.pack(self.w2, self.w2_8)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """x: bf16 [rows][width].  Keeps x, norm(x) and the hidden layer in 8 bits.  Returns the block's own buffer, which the
        next call writes."""
        layers.pack(x, self.x8)
        layers.layer_norm(x, self.gamma, self.beta, EPS, self.mean, self.rstd, packed=self.h8)
        layers.product(self.h8, self.w1_8, packed=self.a8, slope=SLOPE)
        layers.product(self.a8, self.w2_8, y=self.y)
        return self.y.add_(x)

    def backward(self, dy: torch.Tensor, node_start: Optional[torch.Tensor] = None) -> torch.Tensor:
        """dy: bf16 [rows][width], the gradient at y.  Every node's gradients go to its row of `grads`; returns the gradient at
        x, in the block's own buffer, which the next call writes."""
        at, g = self.at, self.grads
        layers.pack(dy, self.dy8)
        layers.weight_gradient(dy, self.a8, g[:, at[3]:at[4]], node_start=node_start)
        layers.product(self.dy8, self.w2_8, y=self.da, across=True)
        layers.pack(self.da, self.dz8, slope=SLOPE, gate=self.a8, y=self.dz)
        layers.weight_gradient(self.dz, self.h8, g[:, at[2]:at[3]], node_start=node_start)
        layers.product(self.dz8, self.w1_8, y=self.dh, across=True)
        layers.layer_norm_backward(self.dh, self.x8, self.gamma, self.mean, self.rstd, self.dx, g[:, at[0]:at[1]], g[:, at[1]:at[2]],
                                   node_start=node_start)
        return self.dx.add_(dy)


def train(block: ResidualBlock, steps: int, lr: float = 0.0, density_ppm: int = 20000, seed: int = 1, say=None):
    """Fits the block to a fixed random map, its gradients compressed at every step: the norm's parameters are sent as they
    are, of the weights' gradients the largest entries with error feedback.  lr: 0 selects 1 / hidden (the curvature grows
    with the number of hidden units).  Returns the losses."""
    lr = lr or 1.0 / block.hidden
    dev = block.theta.device
    ctx = lgc.LGC(block.numel, block.K, density_ppm=density_ppm, momentum=0.5, ae_kind="identity", layer_mode=["dense", "dense", "ae", "ae"], device=dev)
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    target = torch.randn(block.width, block.width, generator=g, device=dev) * block.width ** -0.5
    start = torch.linspace(0, block.rows, block.K + 1, device=dev).long()
    update, losses = torch.empty(block.N, device=dev), []
    for step in range(steps):
        x = torch.randn(block.rows, block.width, generator=g, device=dev).bfloat16()
        d = block.forward(x).float() - (x.float() + torch.tanh(x.float() @ target))
        losses.append(d.square().mean())
        block.backward((d * (2.0 * block.K / block.rows)).bfloat16(), start)      # every node's mean over its rows
        ctx.step(block.grads, update, step % block.K)
        block.theta.sub_(update, alpha=lr)
        block.refresh()
        if say and step % 10 == 0:
            say(f"step {step:4d}  loss {losses[-1].item():.4f}")
    ctx.check()
    layers.check()
    return torch.stack(losses)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("nodes", 4), ("rows", 4096), ("width", 1024), ("hidden", 4096), ("steps", 40)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    block = ResidualBlock(a.rows, a.width, a.hidden, a.nodes)
    losses = train(block, a.steps, say=print)
    print(f"{a.steps} steps: loss {losses[0].item():.4f} -> {losses[-1].item():.4f}")
    x = torch.randn(a.rows, a.width, device="cuda").bfloat16()
    dy = torch.randn(a.rows, a.width, device="cuda").bfloat16()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start = torch.linspace(0, a.rows, a.nodes + 1, device="cuda").long()
    for timed in (False, True):
        begin.record()
        for _ in range(10):
            block.forward(x)
            block.backward(dy, start)
        end.record()
        torch.cuda.synchronize()
    print(f"forward and backward: {begin.elapsed_time(end) / 10:.3f} ms")


if __name__ == "__main__":
    main()
