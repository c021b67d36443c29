"""GPU parity of the dropout with the fp64 oracle: the mask bit for bit, the values to two roundings in fp32 and one of the result."""
import numpy as np
import pytest
import torch

from oracle import epilogue as oep

pytestmark = pytest.mark.gpu
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("T,D", [(1, 1), (1, 7), (1, 8), (3, 9), (5, 1000), (257, 24), (64, 4096), (7, 4099), (2000, 3)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.99])
def test_dropout(metis, T, D, dtype, p):
    g = torch.Generator().manual_seed(T + D)
    x, r = torch.randn((T, D), generator=g).to(dtype), torch.randn((T, D), generator=g).to(dtype)
    seed = 0xFEDCBA9876543210
    step = torch.tensor([123456789012], dtype=torch.int64, device="cuda")
    m = oep.mask(p, seed, 123456789012, np.arange(T), D)
    mask = metis.DropoutMask(p, seed, step)
    for pad, where in ((0, "new"), (3, "new"), (1, "x"), (0, "residual")):
        whole = [torch.full((T, D + 2 * pad), 7.0, dtype=dtype, device="cuda") for _ in range(3)]
        xd, rd, y = (t[:, pad:pad + D] for t in whole)
        xd.copy_(x)
        rd.copy_(r)
        for res in (None, rd):
            if where == "residual" and res is None:
                continue
            out = {"new": y, "x": xd, "residual": rd}[where]
            assert metis.dropout(xd, out, mask, residual=res) is out
            a = m * x.double().numpy()
            b = r.double().numpy() if res is not None else 0.0
            got, ref = out.double().cpu().numpy(), a + b
            assert np.all(np.abs(got - ref) <= 3 * 2.0 ** -24 * (np.abs(a) + np.abs(b)) + ROUND[dtype] * np.abs(ref) * 1.001)
            if res is None:
                assert (got[m == 0] == 0).all()
            xd.copy_(x)
            rd.copy_(r)
        for t in whole:
            assert (t[:, :pad] == 7).all() and (t[:, pad + D:] == 7).all()


def test_mask_is_of_the_element_alone(metis):
    """Types, strides and the product's epilogue see the same mask, and the backward pass is the forward pass's call."""
    T, D = 70, 203
    mask = metis.DropoutMask(0.3, 5)
    ones = torch.ones((T, D), device="cuda")
    a = metis.dropout(ones, torch.empty_like(ones), mask)
    assert np.array_equal(a.cpu().numpy().astype(np.float64) > 0, oep.mask(0.3, 5, 0, np.arange(T), D) > 0)
    b = metis.dropout(ones.to(torch.bfloat16), torch.empty((T, D), dtype=torch.bfloat16, device="cuda"), mask)
    assert torch.equal(a > 0, b > 0)
    W = metis.quantize_mx(torch.zeros((D, 32), device="cuda"), metis.MxTensor(D, 32))
    c = metis.mxfp4_linear(torch.zeros((T, 32), device="cuda"), W, torch.empty((T, D), device="cuda"), bias=torch.ones(D, device="cuda"), mask=mask)
    assert torch.equal(a, c)
    d = metis.linear_grads(ones, torch.empty_like(ones), mask=mask)
    assert torch.equal(a, d)


def test_missing_values_are_dropped(metis):
    x = torch.full((4, 100), float("nan"), device="cuda")
    x[1:] = float("inf")
    y = metis.dropout(x, torch.empty_like(x), metis.DropoutMask(0.5, 1), residual=torch.ones_like(x)).cpu().numpy()
    m = oep.mask(0.5, 1, 0, np.arange(4), 100)
    assert (y[m == 0] == 1).all() and not np.isfinite(y[m > 0]).any()


def test_a_captured_dropout_follows_the_step(metis):
    x = torch.randn((50, 333), device="cuda")
    y, step = torch.empty_like(x), torch.zeros(1, dtype=torch.int64, device="cuda")
    mask = metis.DropoutMask(0.4, 17, step)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        metis.dropout(x, y, mask)
        step.add_(1)
    torch.cuda.synchronize()
    for i in range(4):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(y.cpu().numpy() != 0, oep.mask(0.4, 17, i, np.arange(50), 333) > 0), i
        assert torch.randn((64, 64), device="cuda").isfinite().all()


def test_no_rows(metis):
    e = torch.empty((0, 5), device="cuda")
    metis.dropout(e, e, metis.DropoutMask(0.1, 1))
