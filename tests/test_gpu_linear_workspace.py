"""What a product of rows that are quantized already allocates: the sums of its contraction's parts, and nothing where it is not cut."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("T,N,K,cut", [(4352, 4112, 512, False), (300, 520, 512, False), (64, 520, 4096, False), (128, 1024, 4096, True), (129, 777, 2080, True)])
def test_allocations(metis, T, N, K, cut):
    x, w = torch.randn((T, K), device="cuda"), torch.randn((N, K), device="cuda")
    X, W = metis.quantize_mx(x, metis.MxTensor(T, K)), metis.quantize_mx(w, metis.MxTensor(N, K))
    Y = torch.empty((T, N), device="cuda")
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    metis.mxfp4_linear(X, W, Y)
    taken = torch.cuda.max_memory_allocated() - before
    need = metis.mxfp4_linear_workspace_bytes(T, N, K, quantized=True)
    assert (need > 0) == cut and need <= taken <= need + 512
    if cut:                                                          # several parts' sums in fp32
        assert need >= 2 * 4 * T * N and need % (4 * 64) == 0 and need < metis.mxfp4_linear_workspace_bytes(T, N, K)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        assert torch.equal(metis.mxfp4_linear(X, W, torch.empty_like(Y), workspace=ws), Y)
