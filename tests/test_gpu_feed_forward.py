"""The operators around the products as they are used together: a pre-norm feed-forward block forward and backward, replayed from a graph, on another
stream, and one token at a time."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import epilogue as oep
from oracle import mx as omx

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("feed_forward_block", os.path.join(ROOT, "examples", "feed_forward_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert torch.cuda.is_available()
    m.metis.lib()
    return m


def _f64(t):
    return t.double().cpu().numpy()


def _q(x):
    return omx.dequantize_mx(*omx.quantize_mx(x))


def _block(example, act="gelu", p=0.2, T=96, D=128, F=320):
    b = example.FeedForwardBlock(D, F, p, act, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda")
    b.up_bias.copy_(0.3 * draw(F))
    b.down_bias.copy_(0.3 * draw(D))
    b.gain.add_(0.2 * draw(D))
    b.shift.copy_(0.2 * draw(D))
    b.step_number.fill_(41)
    return b, draw(T, D).to(torch.bfloat16), draw(T, D).to(torch.bfloat16)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
def test_forward_and_backward(example, act):
    """Every operator on what the one before it left (so that a code next to a border does not decide), to bf16's rounding 2^-8 of the result and as much of
    what an fp32 sum of the row's products may be off, K 2^-24 of their magnitudes, and 1e-4 for what the activations add."""
    b, x, dy = _block(example, act)
    y, kept = b.forward(x)
    _, stats, h, pre, a = kept
    near = lambda got, ref, big: np.testing.assert_array_less(np.abs(_f64(got) - ref), 2.0 ** -8 * np.abs(ref) + 3e-4 * big + 1e-30)
    hr, sr = oep.layernorm(_f64(x), _f64(b.gain), _f64(b.shift), 1e-5)
    near(h, hr, 1e-2)
    W1, W2, X1, X2 = _q(_f64(b.up)), _q(_f64(b.down)), _q(_f64(h)), _q(_f64(a))
    z = X1 @ W1.T + _f64(b.up_bias)
    big = np.abs(X1) @ np.abs(W1).T + 1
    near(pre, z, big)
    near(a, oep.act(act, z), big)
    m = oep.mask(b.p, 4, 41, np.arange(96), 128)
    near(y, _f64(x) + m * (X2 @ W2.T + _f64(b.down_bias)), np.abs(X2) @ np.abs(W2).T + np.abs(_f64(x)) + 1)
    # the backward pass in one go, straight through the quantizers.  Each product's operands are rounded to a mantissa bit (values spread over a binade are
    # off by up to a quarter, 0.13 in the root of the mean square at most), two a product and two products on the longest way: 0.13 * 2 = 0.26
    dx, g = b.backward(dy, kept)
    d = m * _f64(dy)
    da = d @ _f64(b.down)
    dz = da * sum(oep.slope_terms(act, _f64(pre)))
    dh = dz @ _f64(b.up)
    rdx, rgain, rshift = oep.layernorm_grads(dh, _f64(x), _f64(stats), _f64(b.gain), _f64(dy))
    ref = dict(down_bias=d.sum(0), up_bias=dz.sum(0), down=d.T @ _f64(a), up=dz.T @ _f64(h), gain=rgain, shift=rshift)
    for name, r in ref.items():
        assert np.linalg.norm(_f64(g[name]) - r) <= (1e-5 if name == "down_bias" else 0.26) * np.linalg.norm(r), name
    assert np.linalg.norm(_f64(dx) - rdx) <= 0.26 * np.linalg.norm(rdx - _f64(dy)) + 2.0 ** -8 * np.linalg.norm(rdx)


def _step(b, x, dy):
    y, kept = b.forward(x)
    dx, g = b.backward(dy, kept)
    return [y, dx] + [g[k] for k in sorted(g)]


def test_a_captured_step_replays(example):
    """Graphs of two blocks, replayed in turns with eager work between them: every replay gives the bits of the eager step with the same number."""
    made = []
    for p, T, D, F in ((0.2, 96, 128, 320), (0.3, 640, 256, 1024)):
        b, x, dy = _block(example, "gelu", p, T, D, F)
        eager = []
        for i in range(4):
            b.step_number.fill_(i)
            eager.append([t.clone() for t in _step(b, x, dy)])
        assert not torch.equal(eager[0][0], eager[1][0])                # another mask
        b.step_number.fill_(0)
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            outs = _step(b, x, dy)
            b.step_number.add_(1)
        made.append((graph, outs, eager, (b, x, dy)))           # (what a graph reads has to live as long as it)
    torch.cuda.synchronize()
    for i in range(4):
        for graph, outs, eager, _ in made:
            for t in outs:
                t.zero_()
            assert (torch.randn((256, 256), device="cuda") @ torch.randn((256, 256), device="cuda")).isfinite().all()
            graph.replay()
        torch.cuda.synchronize()
        for graph, outs, eager, _ in made:
            for k, (t, e) in enumerate(zip(outs, eager[i])):
                assert torch.equal(t, e), (i, k)


def test_two_streams(example):
    """The same step on two streams at once, each with tensors of its own, gives the bits of a step alone."""
    blocks = [_block(example, "silu", 0.2, 320, 256, 768) for _ in range(2)]
    ref = [t.clone() for t in _step(*blocks[0])]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(3):
        for s, (b, x, dy) in zip(streams, blocks):
            with torch.cuda.stream(s):
                outs.append(_step(b, x, dy))
    torch.cuda.synchronize()
    for o in outs:
        for t, r in zip(o, ref):
            assert torch.equal(t, r)


def test_single_tokens_and_prompts(example):
    """Served in any grouping, a token's row is the same to a rounding of bf16 here and there (sums in another order), which may move a code of the next
    product's row by one: 2^-8 for what is not moved, and a fifth of the elements moved by a quarter of a row's share each would be 5e-3."""
    b, x, _ = _block(example, "gelu", 0.2, 200, 256, 1024)
    y = b.forward(x, training=False)[0].double()
    for cut in ([1] * 8 + [192], [64, 65, 71], [17, 33, 150]):
        got = torch.cat([b.forward(p, training=False)[0] for p in x.split(cut)]).double()
        assert (got - y).norm() <= 2e-2 * y.norm()


def test_example_runs(example):
    losses, block, x, batch = example.main(["--tokens", "256", "--hidden", "128", "--inner", "256", "--steps", "4"])
    assert len(losses) == 4 and all(np.isfinite(losses)) and batch.shape == x.shape
