"""The mixture-of-experts calls write their outputs and workspaces and nothing else, where launches have more workgroups than there is work for."""
import numpy as np
import pytest
import torch

from oracle import mx as omx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def _guarded(n, guard):
    """a buffer of n bytes, and the bytes behind it"""
    whole = torch.full((n + guard,), 0xA5, dtype=torch.uint8, device="cuda")
    return whole[:n], whole[n:]


@pytest.mark.parametrize("groups,M,N", [(32769, 32, 8), (40000, 32, 8), (130, 64544, 8), (1, 8389120, 8)])
def test_quantize_mx_t_of_more_units_than_a_grid_axis_takes(metis, groups, M, N):
    """More than 32768 units of 256 rows, which no longer lie along one axis of the grid."""
    assert groups * -(-M // 256) > 32768
    x = torch.randn((groups * M, N), generator=torch.Generator(device="cuda").manual_seed(groups), device="cuda").to(torch.bfloat16)
    n = groups * M * N
    (codes, codes_end), (scales, scales_end) = _guarded(n // 2, 65536 * 256 * N // 2), _guarded(n // 32, 65536 * 256 * N // 32)
    metis.quantize_mx_t(x, metis.MxTensor(groups * N, M, buffers=(codes, scales)), groups)
    want = metis.quantize_mx(x.view(groups, M, N).transpose(1, 2).contiguous().view(groups * N, M), metis.MxTensor(groups * N, M))
    assert torch.equal(codes, want.codes.flatten()) and torch.equal(scales, want.scales.flatten())
    assert bool((codes_end == 0xA5).all()) and bool((scales_end == 0xA5).all())
    m = min(M, 8192)                                           # the last rows of the last group, by the oracle
    c, s = omx.quantize_mx(x[-m:].double().cpu().numpy().T)
    assert np.array_equal(codes.view(groups * N, -1)[-N:, -m // 2:].cpu().numpy(), c)
    assert np.array_equal(scales.view(groups * N, -1)[-N:, -m // 32:].cpu().numpy(), s)
