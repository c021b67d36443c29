"""One expert that has every token once: the streamed product gives the bits of the dense streamed product of the same operands.  Both multiply the
same blocks by the same instruction in the same order and round once, so no tolerance is due.  (Sizes: more than 128 tiles of 256 x 256, so that
the contraction is not cut into parts, and eight units of 256 at least, where the dense product streams too.  A smaller product goes straight from
memory, in another order.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,N,K", [(3000, 3400, 2048), (4100, 2600, 2304)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_streamed_product_of_one_expert_is_the_dense_one(T, N, K, out):
    from paper_2509_00404_amd import metis
    g = torch.Generator(device="cuda").manual_seed(T)
    x, w = (torch.randn((n, K), generator=g, device="cuda").to(torch.bfloat16) for n in (T, N))
    X, W = metis.quantize_mx(x, metis.MxTensor(T, K)), metis.quantize_mx(w, metis.MxTensor(N, K))
    want = metis.mxfp4_gemm_nt(X, W, torch.empty((T, N), dtype=out, device="cuda"))
    plan = metis.dispatch(torch.zeros((T, 1), dtype=torch.int32, device="cuda"), 1)
    for gather in (False, True):
        got = torch.full((T, N), float("nan"), dtype=out, device="cuda")
        metis.experts_product(x, W, plan, got, gather=gather)
        assert torch.equal(got, want)
