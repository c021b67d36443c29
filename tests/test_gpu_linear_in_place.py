"""Outputs of the linear layer in the place of the rows it reads: where those are quantized by a launch of their own, the same bits as beside them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("T,N", [(17, 64), (33, 1024), (100, 544), (128, 4096), (300, 2080), (4352, 4352), (4100, 4096)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_outputs_over_rows(metis, T, N, dtype):
    g = torch.Generator(device="cuda").manual_seed(T)
    x, w = (torch.randn(s, generator=g, device="cuda") for s in ((T, N), (N, N)))
    x, W, bias = x.to(dtype), metis.quantize_mx(w * N ** -0.5, metis.MxTensor(N, N)), torch.randn(N, generator=g, device="cuda")
    assert metis.mxfp4_linear_workspace_bytes(T, N, N) > 0
    e = dict(bias=bias, act="gelu", mask=metis.DropoutMask(0.2, 3))
    y, pre = torch.empty_like(x), torch.empty_like(x)
    metis.mxfp4_linear(x, W, y, pre=pre, residual=x, **e)
    a = x.clone()
    assert torch.equal(metis.mxfp4_linear(a, W, a, residual=a, **e), y)
    a, b = x.clone(), torch.empty_like(x)
    metis.mxfp4_linear(a, W, b, pre=a, residual=x, **e)
    assert torch.equal(a, pre) and torch.equal(b, y)


def test_refused_where_rows_are_quantized_on_the_spot(metis):
    x, W = torch.randn((4, 64), device="cuda"), metis.quantize_mx(torch.randn((64, 64), device="cuda"), metis.MxTensor(64, 64))
    kept = x.clone()
    for kw in (dict(Y=x), dict(Y=torch.empty_like(x), pre=x)):
        with pytest.raises(metis.MetisError):
            metis.mxfp4_linear(x, W, **kw)
    assert torch.equal(x, kept)
    wide = torch.zeros((4, 128), device="cuda")                      # rows and outputs side by side in one buffer
    wide[:, :64] = x
    assert torch.equal(metis.mxfp4_linear(wide[:, :64], W, wide[:, 64:]), metis.mxfp4_linear(x, W, torch.empty_like(x)))
