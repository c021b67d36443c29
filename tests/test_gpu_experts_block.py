"""The example block: its steps learn, its gradients are those of the quantized forward's own chain, and single tokens are served as in a batch.

Gradients: MXFP4 rounds every operand of every product to about 0.1 of its size, independently from element to element, so a gradient computed
in fp64 from the unquantized weights points the same way within a few tenths (cosine above 0.9) and no closer.  A token alone takes other
kernels than in a batch: fp32 sums in another order, some bf16 roundings and FP4 codes the other way -> 1e-2 relative."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available()
    spec = importlib.util.spec_from_file_location("experts_block", os.path.join(ROOT, "examples", "experts_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_steps_learn_and_single_tokens_agree(example):
    losses, block, x, batch = example.main(["--tokens", "512", "--hidden", "256", "--inner", "128", "--experts", "8", "--choices", "2", "--steps", "20"])
    assert losses[-1] < 0.9 * losses[0]
    one = torch.cat([block.forward(x[t:t + 1], training=False)[0] for t in range(8)]).float()
    assert float((one - batch[:8].float()).norm() / batch[:8].float().norm()) < 1e-2


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_gradients_point_the_right_way(example, scores):
    T, D, F, E, k = 300, 256, 128, 8, 2
    block = example.ExpertsBlock(D, F, E, k, seed=5, scores=scores)
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((T, D), generator=g, device="cuda").to(torch.bfloat16)
    dy = torch.randn((T, D), generator=g, device="cuda").to(torch.bfloat16)
    y, kept = block.forward(x)
    grads = block.backward(dy, kept)
    # the same block in fp64 on the CPU, the choices as they were made
    leaves = [t.detach().double().cpu().requires_grad_(True) for t in (x, block.router, block.up, block.down)]
    xr, router, up, down = leaves
    idx = kept[2].cpu().long()
    logits = xr @ router.t()
    s = torch.sigmoid(logits) if scores == "sigmoid" else torch.softmax(logits, 1)
    w = s.gather(1, idx)
    w = w / w.sum(1, keepdim=True)
    out = 0
    for j in range(k):
        gu = torch.einsum("td,tfd->tf", xr, up.view(E, 2 * F, D)[idx[:, j]])
        act = torch.nn.functional.silu(gu[:, :F]) * gu[:, F:]
        out = out + w[:, j, None] * torch.einsum("tf,tdf->td", act, down.view(E, D, F)[idx[:, j]])
    ref = torch.autograd.grad(out, leaves, dy.double().cpu())
    cos = torch.nn.functional.cosine_similarity
    assert float(cos(y.double().cpu().flatten(), out.detach().flatten(), dim=0)) > 0.95
    for name, got, want in zip(("x", "router", "up", "down"), grads, ref):
        c = float(cos(got.double().cpu().flatten(), want.flatten(), dim=0))
        assert c > 0.9, (name, c)
