"""A ring of replicas trains a residual network of gated feed-forward blocks on a synthetic regression.

Every replica has weights and data of its own; all of them live on one GPU, and every call works on all of them:

    residual_norm -> feed_forward -> residual_norm -> ... -> loss
    ... backward of the same, gradients straight into the layout that the step reads ...
    clip_gradients (16-bit gradients -> fp32)  ->  EventGrad.step

The fp32 parameters are the step's; forward and backward work on a copy in the compute type.

    python examples/residual_ffn_ring.py --replicas 4 --blocks 2 --steps 100
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2103_07454_b200 import binding as B  # noqa: E402

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


class Network:
    """P copies of: a norm, then `blocks` times (feed-forward block, norm with gate and scaled residual)."""

    def __init__(self, P: int, blocks: int, width: int, hidden: int, dtype: torch.dtype, horizon: float = 1.0):
        self.P, self.blocks, self.width, self.hidden, self.dtype = P, blocks, width, hidden, dtype
        # w_pre of the first norm; then, block by block, gate / up / down projection, w_post, gate, scale, w_pre
        self.shapes = [(width,)]
        for _ in range(blocks):
            self.shapes += [(hidden, width), (hidden, width), (width, hidden)] + [(width,)] * 4
        numel = [s[0] * (s[1] if len(s) == 2 else 1) for s in self.shapes]
        self.ring = B.EventGrad(P, numel, horizon=horizon)
        self.ring.set_carry_norm(True)
        self.params = self.ring.empty_params()
        self.work = torch.zeros_like(self.params, dtype=dtype)
        self.grads = torch.zeros_like(self.work)
        self.grads32 = self.grads if dtype is torch.float32 else torch.zeros_like(self.params)

    def view(self, buffer: torch.Tensor, t: int) -> torch.Tensor:
        return self.ring.view(buffer, t, self.shapes[t])

    def initialise(self, seed: int):
        """The same start for every replica."""
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for t, shape in enumerate(self.shapes):
            v = self.view(self.params, t)
            if len(shape) == 2:
                v.copy_((torch.randn(shape, generator=gen, device="cuda") * shape[1] ** -0.5).expand_as(v))
            else:
                v.fill_(0.0 if self.is_gate(t) else 1.0)
        self.work.copy_(self.params)

    def is_gate(self, t: int) -> bool:
        return t > 0 and (t - 1) % 7 == 4

    def weights(self, buffer: torch.Tensor, block: int):
        """((gate, up, down), (w_post, gate, scale, w_pre)) of a block."""
        at = 1 + 7 * block
        return tuple(self.view(buffer, at + q) for q in range(3)), tuple(self.view(buffer, at + q) for q in range(3, 7))

    def forward(self, x: torch.Tensor):
        """(output, what the backward pass needs) for ``x`` of ``[P, tokens, width]``."""
        r, o = B.residual_norm(None, x, w_pre=self.view(self.work, 0))
        kept = []
        for l in range(self.blocks):
            ffn, (w_post, gate, scale, w_pre) = self.weights(self.work, l)
            y, saved = B.feed_forward(o, *ffn, save=True)
            kept.append((o, saved, y, r))
            r, o = B.residual_norm(y, r, w_post=w_post, gate=gate, scale=scale, w_pre=w_pre)
        return o, kept

    def backward(self, x: torch.Tensor, kept, d_o: torch.Tensor):
        """Gradients of all weights into ``self.grads`` from the gradient of the output."""
        d_r = None
        for l in reversed(range(self.blocks)):
            o, saved, y, r = kept[l]
            ffn, (w_post, gate, scale, w_pre) = self.weights(self.work, l)
            d_ffn, d_norm = self.weights(self.grads, l)
            dy, d_r, _ = B.residual_norm_backward(d_r, d_o, y, r, w_post=w_post, gate=gate, scale=scale, w_pre=w_pre,
                                                  d_weights=d_norm)
            d_o, _ = B.feed_forward_backward(dy, o, *ffn, saved, d_weights=d_ffn)
        B.residual_norm_backward(d_r, d_o, None, x, w_pre=self.view(self.work, 0),
                                 d_weights=(None, None, None, self.view(self.grads, 0)))

    def step(self, lr: float, max_norm: float) -> torch.Tensor:
        """Clips, exchanges what has changed enough, averages, updates; the gradients' norms before clipping."""
        norms = self.ring.clip_gradients(self.grads, max_norm, out=self.grads32, zero_nonfinite=True)
        self.ring.step(self.params, self.grads32, lr)
        self.work.copy_(self.params)
        return norms


def batch(P: int, tokens: int, width: int, seed: int, dtype: torch.dtype):
    """Inputs of every replica and the targets of a fixed teacher."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((P, tokens, width), generator=gen, device="cuda")
    teacher = torch.randn((width, width), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * width ** -0.5
    return x.to(dtype), torch.tanh(x @ teacher)


def train(replicas=4, blocks=2, width=64, hidden=176, tokens=128, steps=100, lr=0.5, max_norm=1.0, dtype="bf16", report=0):
    """Mean loss of the replicas, step by step, and the share of messages that were sent."""
    dt = TYPES[dtype]
    net = Network(replicas, blocks, width, hidden, dt)
    net.initialise(0)
    losses = []
    for k in range(steps):
        x, target = batch(replicas, tokens, width, 100 + k, dt)
        out, kept = net.forward(x)
        diff = out.float() - target
        losses.append(diff.pow(2).mean())
        net.backward(x, kept, (diff * (2.0 / (tokens * width))).to(dt))
        norms = net.step(lr, max_norm)
        if report and (k + 1) % report == 0:
            sent = net.ring.stats()["messages"] / (replicas * len(net.shapes) * min(2, max(1, replicas - 1)) * (k + 1))
            print(f"step {k + 1}: loss {float(losses[-1]):.4f}, largest gradient norm {float(norms.max()):.3f}, "
                  f"{100 * sent:.0f} % of the messages sent")
    if B.operator_status() != 0:
        raise B.EventGradError("a bounded wait ran out")
    sent = net.ring.stats()["messages"] / (replicas * len(net.shapes) * min(2, max(1, replicas - 1)) * steps)
    return [float(v) for v in losses], sent


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("replicas", 4), ("blocks", 2), ("width", 64), ("hidden", 176), ("tokens", 128), ("steps", 100)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--dtype", choices=sorted(TYPES), default="bf16")
    a = ap.parse_args()
    losses, sent = train(a.replicas, a.blocks, a.width, a.hidden, a.tokens, a.steps, a.lr, a.max_norm, a.dtype,
                         report=max(1, a.steps // 10))
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}, {100 * sent:.0f} % of the messages sent")
