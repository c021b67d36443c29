"""Shapes that reach the instances of the linear layer's kernels one by one: against the fp64 oracle, with the bounds of test_gpu_linear_epilogue."""
import pytest
import torch

from test_gpu_linear_epilogue import EPILOGUES, _Layer, metis  # noqa: F401  (metis: the fixture)

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,N,K", [(1, 8192, 1024), (13, 8200, 2080), (16, 14336, 544), (17, 8193, 1056), (24, 14336, 1024), (32, 8200, 96), (33, 8195, 2080),
                                   (64, 8192, 4096), (64, 14336, 512), (5, 10000, 5120)])
def test_few_rows_of_many_outputs(metis, T, N, K, dtype):
    """Up to 64 rows, 32 outputs a workgroup; rows quantized already, by a launch of their own, and on the spot."""
    layer = _Layer(metis, T, N, K, dtype, T + N)
    for e in EPILOGUES:
        layer.check(**e)
    layer.check(act="gelu", p=0.2, residual=True, pre=True, pad=3)
    layer.check(act="gelu", p=0.2, residual=True, pre=True, pad=1, dense=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,N,K", [(4352, 4112, 512), (4352, 4096, 768), (2050, 8192, 2048)])
def test_streamed_products_of_every_activation(metis, T, N, K, dtype):
    layer = _Layer(metis, T, N, K, dtype, K)
    for act in ACTS:
        layer.check(act=act)
        layer.check(act=act, pre=True, p=0.1, residual=True)
        layer.check(act=act, bias=False, inplace=True, pre=True, pad=1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,N,K", [(4096, 4096, 256), (4096, 4096, 1024), (4000, 4001, 1024), (3000, 3001, 512)])
def test_whole_stages_in_large_tiles(metis, T, N, K, dtype):
    layer = _Layer(metis, T, N, K, dtype, K)
    for act in ACTS:
        layer.check(act=act, pre=True, p=0.1, residual=True)
    layer.check(act="gelu", dense=True, pad=3)
    layer.check(bias=False, inplace=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,N,K", [(100, 200, 384), (300, 1000, 384), (257, 520, 640), (129, 1024, 2176), (300, 2056, 2176), (65, 64, 2176), (128, 300, 4224)])
def test_contractions_that_end_half_a_unit(metis, T, N, K, dtype):
    """K = 128 beyond whole units of 256, scale rows of whole words: several units, whole and cut into parts."""
    layer = _Layer(metis, T, N, K, dtype, T + N)
    for e in EPILOGUES:
        layer.check(pad=3 if "p" in e else 0, **e)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,N,K", [(128, 1024, 4096), (129, 777, 2080), (65, 64, 2176), (300, 520, 512), (1000, 264, 4096), (200, 100, 14336), (40, 300, 1056)])
def test_any_workspace(metis, T, N, K, dtype):
    """Rows quantized already: without a workspace, with one that holds no numbers, and with too little of one, the same up to the order of the parts'
    sums.  Dense rows: a workspace that holds no numbers."""
    layer = _Layer(metis, T, N, K, dtype, T + N)
    need = metis.mxfp4_linear_workspace_bytes(T, N, K)
    e = dict(act="silu", p=0.2, residual=True, pre=True)
    layer.check(workspace=torch.empty(0, dtype=torch.uint8, device="cuda"), **e)
    a = layer.check(workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"), **e)
    assert torch.equal(a, layer.check(**e))
    layer.check(workspace=torch.full((max(need // 64 - 256, 256),), 255, dtype=torch.uint8, device="cuda"), **e)
    b = layer.check(workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"), dense=True, **e)
    assert torch.equal(b, layer.check(dense=True, **e))
