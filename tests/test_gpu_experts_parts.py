"""GPU parity of the experts' products whose contraction is cut into parts (few tiles, long contractions) with the oracle's fp64 products, at the
bounds of test_gpu_experts: every product is exact in fp32, and parts add up in fewer roundings in a row than the whole."""
import numpy as np
import pytest
import torch

from oracle import experts as oe
from oracle import mx as omx
from test_gpu_experts import _check, _codes, _dense, _plan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


CASES = [  # T, E, k, N, K, skew, missing
    (600, 4, 2, 514, 4096, 0.0, 0.0),
    (300, 2, 1, 513, 14304, 0.0, 0.0),                         # as many parts as there are at most, the last unit short
    (900, 8, 2, 330, 3680, 0.8, 0.2),                          # an expert without slots, slots without an expert
    (2100, 1, 1, 344, 3104, 0.0, 0.0),                          # the last part's units fewer; a unit of one block
    (2000, 4, 4, 33, 8352, 0.0, 0.0),
    (640, 3, 2, 400, 4640, 0.0, 1.0),                          # nobody has an expert
    (5000, 120, 6, 64, 4096, 0.9, 0.0),                        # more tiles than the chip has CUs
]


@pytest.mark.parametrize("T,E,k,N,K,skew,missing", CASES)
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
def test_product_in_parts(metis, T, E, k, N, K, skew, missing, gather, dtype, out):
    if T == 5000 and not gather:
        pytest.skip("the oracle would take the rows of every slot")
    plan, g = _plan(metis, T, E, k, T + N, skew, missing)
    x, w = _dense(g, T if gather else T * k, K, dtype), _dense(g, E * N, K, torch.bfloat16)
    W = metis.MxTensor(E * N, K)
    metis.quantize_mx(w.cuda(), W)
    offsets, token = plan.offsets.cpu().numpy(), plan.token.cpu().numpy()
    ref = oe.experts_product(x.double().numpy(), _codes(W), offsets, token, gather)
    big = oe.experts_product(x.double().abs().numpy(), omx.quantize_mx(np.abs(omx.dequantize_mx(*_codes(W)))), offsets, token, gather)
    need = metis.experts_workspace_bytes(x.shape[0], T * k, E, N, K)
    before = None
    for pad in (0, 3, 0):
        ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")             # (NaN, wherever it is read before it is written)
        C = torch.full((T * k, N + pad), float("nan"), dtype=out, device="cuda")
        metis.experts_product(x.cuda(), W, plan, C[:, pad:], gather=gather, workspace=ws[:need])
        _check(C[:, pad:], ref, big, out)
        assert torch.isnan(C[:, :pad]).all() and bool((ws[need:] == 255).all())
        assert not C[int(offsets[-1]):, pad:].any()
        assert before is None or torch.equal(before, C[:, pad:])
        before = C[:, pad:].clone()


def test_in_a_graph(metis):
    T, E, k, N, K = 256, 16, 4, 1024, 4096
    plan, g = _plan(metis, T, E, k, 5)
    x, w = _dense(g, T, K, torch.bfloat16).cuda(), _dense(g, E * N, K, torch.bfloat16)
    W = metis.MxTensor(E * N, K)
    metis.quantize_mx(w.cuda(), W)
    C = torch.empty((T * k, N), device="cuda")
    ws = torch.empty(metis.experts_workspace_bytes(T, T * k, E, N, K), dtype=torch.uint8, device="cuda")
    run = lambda: metis.experts_product(x, W, plan, C, gather=True, workspace=ws)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        x.copy_(torch.randn((T, K), generator=g).to(torch.bfloat16))
        C.fill_(float("nan"))
        graph.replay()
        got = C.clone()
        torch.cuda.synchronize()
        run()
        assert torch.equal(got, C)
