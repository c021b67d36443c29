"""Workspaces that the Python calls around the products take: device memory, whole, counted in bytes."""
import pytest
import torch


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    return m


def test_host_workspaces(metis):
    """(kernels would follow the host's addresses)"""
    with pytest.raises(AssertionError):
        metis._space(torch.empty(1 << 20, dtype=torch.uint8), 256, None)


@pytest.mark.gpu
def test_workspaces_of_other_types_and_layouts(metis):
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w = torch.randn((128, 4096), generator=g, device="cuda"), torch.randn((256, 4096), generator=g, device="cuda")
    W, Y = metis.quantize_mx(w, metis.MxTensor(256, 4096)), torch.empty((128, 256), device="cuda")
    need = metis.mxfp4_linear_workspace_bytes(128, 256, 4096)
    ref = metis.mxfp4_linear(x, W, Y).clone()
    assert torch.equal(metis.mxfp4_linear(x, W, Y.zero_(), workspace=torch.empty((need + 3) // 4, device="cuda")), ref)
    for bad in (torch.empty(1, dtype=torch.uint8, device="cuda").expand(need), torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(AssertionError):
            metis.mxfp4_linear(x, W, Y, workspace=bad)
    with pytest.raises(metis.MetisError):
        metis.mxfp4_linear(x, W, Y, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
