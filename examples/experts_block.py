"""A mixture-of-experts feed-forward block on the library's MXFP4 products: training steps, and serving one token at a time.

    python examples/experts_block.py                 # trains a small block on a fixed target, then serves single tokens
    python examples/experts_block.py --tokens 16384 --hidden 4096 --inner 1024 --experts 64 --choices 4 --steps 10 --rate 0.01

The block keeps bf16 weights and, beside them, their MXFP4 forms for the two directions: blocks along the contraction of the forward product,
and along that of the input gradient.  What a step keeps for its backward pass is the plan, the 8-bit checkpoint of the gate and up outputs, the
experts' output rows and the router's logits; the activation itself is recomputed from the checkpoint.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_00404_amd import metis  # noqa: E402


class ExpertsBlock:
    """y = sum over a token's chosen experts of weight * W_down (silu(W_gate x) * W_up x)."""

    def __init__(self, hidden, inner, experts, choices, seed=0, scores="softmax"):
        self.D, self.F, self.E, self.k, self.scores = hidden, inner, experts, choices, scores
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda rows, cols: (torch.randn((rows, cols), generator=g, device="cuda") * cols ** -0.5).to(torch.bfloat16)
        self.router = draw(experts, hidden).float()
        self.up = draw(experts * 2 * inner, hidden)             # every expert's gate above its up projection
        self.down = draw(experts * hidden, inner)
        self.bias = torch.zeros((experts,), device="cuda")      # balances the load, in the selection alone
        self.up_q, self.up_t = metis.MxTensor(experts * 2 * inner, hidden), metis.MxTensor(experts * hidden, 2 * inner)
        self.down_q, self.down_t = metis.MxTensor(experts * hidden, inner), metis.MxTensor(experts * inner, hidden)
        self.quantize()

    def quantize(self):
        """After every update of the weights."""
        metis.quantize_mx(self.up, self.up_q)
        metis.quantize_mx(self.down, self.down_q)
        metis.quantize_mx_t(self.up, self.up_t, self.E)
        metis.quantize_mx_t(self.down, self.down_t, self.E)

    def forward(self, x, training=True):
        """x [T, D] bf16 -> y [T, D] bf16, and what the backward pass needs."""
        T, S = x.shape[0], x.shape[0] * self.k
        new = lambda rows, cols: torch.empty((rows, cols), dtype=torch.bfloat16, device=x.device)
        logits = x.float() @ self.router.t()
        idx, weights = metis.route(logits, self.k, bias=self.bias, scores=self.scores)
        plan = metis.dispatch(idx, self.E)
        gate_up = metis.experts_product(x, self.up_q, plan, new(S, 2 * self.F), gather=True)
        saved = metis.Mx8Tensor(S, 2 * self.F) if training else None
        act = metis.swiglu(gate_up, new(S, self.F), saved)
        rows = metis.experts_product(act, self.down_q, plan, new(S, self.D))
        y = metis.combine(rows, plan, new(T, self.D), weights)
        return y, (x, logits, idx, weights, plan, saved, rows) if training else None

    def backward(self, dy, kept):
        """Gradients of x, the router, and the experts' two weights (fp32)."""
        x, logits, idx, weights, plan, saved, rows = kept
        S = rows.shape[0]
        new = lambda r, c, t=torch.bfloat16: torch.empty((r, c), dtype=t, device=x.device)
        drows, dweights = metis.combine_grads(dy, rows, plan, weights)
        dact = metis.experts_product(drows, self.down_t, plan, new(S, self.F))
        dgate_up, act = new(S, 2 * self.F), new(S, self.F)
        metis.swiglu_grads(saved, dact, dgate_up, act)
        ddown = metis.experts_wgrad(drows, act, plan, new(self.E * self.D, self.F, torch.float32))
        dup = metis.experts_wgrad(dgate_up, x, plan, new(self.E * 2 * self.F, self.D, torch.float32), gather=True)
        dx = metis.combine(metis.experts_product(dgate_up, self.up_t, plan, new(S, self.D)), plan, new(x.shape[0], self.D, torch.float32))
        dlogits = metis.route_grads(logits, idx, dweights, scores=self.scores)
        return dx + dlogits @ self.router, dlogits.t() @ x.float(), dup, ddown

    def step(self, x, target, rate):
        """One step of gradient descent on the mean squared error; the loss before it."""
        y, kept = self.forward(x)
        error = y.float() - target
        _, drouter, dup, ddown = self.backward((2.0 / x.shape[0] * error).to(torch.bfloat16), kept)
        self.router -= rate * drouter
        self.up = (self.up.float() - rate * dup).to(torch.bfloat16)
        self.down = (self.down.float() - rate * ddown).to(torch.bfloat16)
        counts = (kept[4].offsets[1:] - kept[4].offsets[:-1]).float()
        self.bias += 1e-3 * torch.sign(counts.mean() - counts)
        self.quantize()
        return error.square().sum(1).mean()


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--tokens", type=int, default=1024)
    p.add_argument("--hidden", type=int, default=512)
    p.add_argument("--inner", type=int, default=256)
    p.add_argument("--experts", type=int, default=16)
    p.add_argument("--choices", type=int, default=4)
    p.add_argument("--steps", type=int, default=30)
    p.add_argument("--rate", type=float, default=0.1)
    a = p.parse_args(argv)
    block = ExpertsBlock(a.hidden, a.inner, a.experts, a.choices)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((a.tokens, a.hidden), generator=g, device="cuda").to(torch.bfloat16)
    target = ExpertsBlock(a.hidden, a.inner, a.experts, a.choices, seed=2).forward(x, training=False)[0].float()
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
