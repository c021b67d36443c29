"""A pre-norm feed-forward block on the library's MXFP4 products: training steps, and serving one token at a time.

    python examples/feed_forward_block.py            # trains a small block on a fixed target, then serves single tokens
    python examples/feed_forward_block.py --tokens 16384 --hidden 4096 --inner 14336 --steps 10 --rate 0.01

y = x + dropout(W2 gelu(W1 norm(x) + b1) + b2).  Bias, activation, dropout and residual happen where the products store; what a step keeps for its
backward pass is the norm's statistics and output, what the activation was applied to, and the activation.  The dropout's mask is never stored: it is
computed again from the layer's seed and the step's number, which lives on the device, so that a captured step draws another mask on every replay.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_00404_amd import metis  # noqa: E402


class FeedForwardBlock:
    def __init__(self, hidden, inner, p=0.1, act="gelu", seed=0):
        self.D, self.F, self.p, self.act = hidden, inner, p, act
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda rows, cols: (torch.randn((rows, cols), generator=g, device="cuda") * cols ** -0.5).to(torch.bfloat16)
        self.up, self.down = draw(inner, hidden), draw(hidden, inner)
        self.up_bias, self.down_bias = torch.zeros((inner,), device="cuda"), torch.zeros((hidden,), device="cuda")
        self.gain, self.shift = torch.ones((hidden,), device="cuda"), torch.zeros((hidden,), device="cuda")
        self.step_number = torch.zeros((1,), dtype=torch.int64, device="cuda")
        self.mask = metis.DropoutMask(p, seed + 1, self.step_number) if p > 0 else None
        self.up_q, self.up_t = metis.MxTensor(inner, hidden), metis.MxTensor(hidden, inner)
        self.down_q, self.down_t = metis.MxTensor(hidden, inner), metis.MxTensor(inner, hidden)
        self.quantize()

    def quantize(self):
        """After every update of the weights: blocks along the contraction of the forward product, and along that of the input gradient."""
        metis.quantize_mx(self.up, self.up_q)
        metis.quantize_mx(self.down, self.down_q)
        metis.quantize_mx_t(self.up, self.up_t)
        metis.quantize_mx_t(self.down, self.down_t)

    def forward(self, x, training=True):
        """x [T, D] bf16 -> y [T, D] bf16, and what the backward pass needs."""
        T = x.shape[0]
        new = lambda cols, t=torch.bfloat16: torch.empty((T, cols), dtype=t, device=x.device)
        stats, pre = (new(2, torch.float32), new(self.F)) if training else (None, None)
        h = metis.layernorm(x, new(self.D), self.gain, self.shift, stats=stats)
        a = metis.mxfp4_linear(h, self.up_q, new(self.F), bias=self.up_bias, act=self.act, pre=pre)
        y = metis.mxfp4_linear(a, self.down_q, new(self.D), bias=self.down_bias, mask=self.mask if training else None, residual=x)
        return y, (x, stats, h, pre, a) if training else None

    def backward(self, dy, kept):
        """Gradients of x (bf16) and of the parameters (fp32).  The weights' gradients contract over the tokens, a multiple of 32."""
        x, stats, h, pre, a = kept
        new = lambda rows, cols, t=torch.bfloat16: torch.empty((rows, cols), dtype=t, device=x.device)
        T, vector = x.shape[0], lambda n: torch.empty((n,), device=x.device)
        turned = lambda m: metis.quantize_mx_t(m, metis.MxTensor(m.shape[1], T))
        g = dict(down_bias=vector(self.D), up_bias=vector(self.F), gain=vector(self.D), shift=vector(self.D))
        d = metis.linear_grads(dy, new(T, self.D), mask=self.mask, dbias=g["down_bias"])
        g["down"] = metis.mxfp4_gemm_nt(turned(d), turned(a), new(self.D, self.F, torch.float32))
        da = metis.mxfp4_linear(d, self.down_t, new(T, self.F))
        dz = metis.linear_grads(da, da, pre=pre, act=self.act, dbias=g["up_bias"])
        g["up"] = metis.mxfp4_gemm_nt(turned(dz), turned(h), new(self.F, self.D, torch.float32))
        dh = metis.mxfp4_linear(dz, self.up_t, new(T, self.D))
        dx = metis.layernorm_grads(dh, x, stats, new(T, self.D), self.gain, g["gain"], g["shift"], add=dy)
        return dx, g

    def step(self, x, target, rate):
        """One step of gradient descent on the mean squared error; the loss before it."""
        y, kept = self.forward(x)
        error = y.float() - target
        _, g = self.backward((2.0 / x.shape[0] * error).to(torch.bfloat16), kept)
        for name, d in g.items():
            p = getattr(self, name)
            p.copy_(p.float() - rate * d)
        self.step_number.add_(1)
        self.quantize()
        return error.square().sum(1).mean()


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--tokens", type=int, default=1024)
    p.add_argument("--hidden", type=int, default=512)
    p.add_argument("--inner", type=int, default=2048)
    p.add_argument("--dropout", type=float, default=0.1)
    p.add_argument("--steps", type=int, default=30)
    p.add_argument("--rate", type=float, default=0.02)
    a = p.parse_args(argv)
    block = FeedForwardBlock(a.hidden, a.inner, a.dropout)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((a.tokens, a.hidden), generator=g, device="cuda").to(torch.bfloat16)
    target = FeedForwardBlock(a.hidden, a.inner, 0.0, seed=2).forward(x, training=False)[0].float()
    losses, t0 = [], None
    for i in range(a.steps):
        if i == 1:
            torch.cuda.synchronize()
            t0 = time.perf_counter()
        losses.append(block.step(x, target, a.rate))
    torch.cuda.synchronize()
    if a.steps > 1:
        print(f"{(time.perf_counter() - t0) / (a.steps - 1) * 1e3:.2f} ms a step")
    print("loss", " ".join(f"{float(v):.4f}" for v in losses[::max(1, a.steps // 10)]), f"-> {float(losses[-1]):.4f}")
    batch = block.forward(x, training=False)[0]
    one = torch.cat([block.forward(x[t:t + 1], training=False)[0] for t in range(4)])
    print("single tokens against the batch, relative:", f"{float((one.float() - batch[:4].float()).norm() / batch[:4].float().norm()):.1e}")
    return [float(v) for v in losses], block, x, batch


if __name__ == "__main__":
    main()
