"""GPU parity of the experts' MXFP4 products with the oracle's fp64 products of the same quantized operands.

Every product of two codes under their scales is exact in fp32, and only the accumulation rounds: 2e-6 relative to the sum of the products'
magnitudes would take 16 roundings in a row at the size of the whole sum; bf16 outputs round once more, 2^-8 relative to the result."""
import numpy as np
import pytest
import torch

from oracle import experts as oe
from oracle import mx as omx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def _plan(metis, T, E, k, seed, skew=0.0, missing=0.0):
    """skew: the share of tokens whose first choice is expert 0, and expert 1 gets none"""
    g = torch.Generator().manual_seed(seed)
    scores = torch.rand((T, E), generator=g)
    if skew and E > 2:
        scores[:, 1] = -1.0
        scores[torch.rand((T,), generator=g) < skew, 0] = 2.0
    idx = torch.topk(scores, k, dim=1).indices
    idx[torch.rand((T, k), generator=g) < missing] = -1
    return metis.dispatch(idx.to(torch.int32).cuda(), E), g


def _dense(g, M, N, dtype, spread=1.0):
    return (torch.randn((M, N), generator=g) * torch.exp(spread * torch.randn((M, 1), generator=g))).to(dtype)


def _check(got, ref, big, out):
    got = got.double().cpu().numpy()
    assert np.all(np.isfinite(got))
    bound = 2e-6 * big + (2.0 ** -8 * np.abs(ref) if out == torch.bfloat16 else 0.0)
    assert np.all(np.abs(got - ref) <= bound + 1e-37)


def _codes(q):
    return q.codes.cpu().numpy().reshape(q.rows, -1), q.scales.cpu().numpy().reshape(q.rows, -1)


CASES = [  # T, E, k, N, K, skew, missing
    (1, 8, 2, 64, 256, 0.0, 0.0),
    (1, 64, 4, 100, 96, 0.0, 0.5),
    (5, 3, 3, 1, 32, 0.0, 0.0),
    (24, 16, 4, 200, 512, 0.5, 0.1),
    (100, 60, 6, 72, 160, 0.9, 0.0),
    (300, 8, 2, 264, 1024, 0.7, 0.2),
    (1000, 4, 1, 520, 544, 0.0, 0.05),
    (700, 4, 2, 513, 768, 0.8, 0.0),
    (2100, 2, 1, 256, 512, 0.0, 0.0),
    (40, 512, 8, 40, 64, 0.0, 0.0),
    (2, 8, 4, 333, 1568, 0.0, 0.0),                            # a decode step, the contraction's last run short
    (9, 8, 2, 1030, 2080, 0.5, 0.1),
    (60, 16, 4, 200, 992, 0.9, 0.0),                           # few slots, too many to quantize on the spot
    (100, 8, 2, 140, 1056, 0.3, 0.0),
    (1100, 4, 2, 520, 160, 0.8, 0.1),                          # enough outputs for the stream, whatever the contraction
    (2200, 2, 1, 513, 544, 0.0, 0.0),
    (900, 60, 6, 203, 96, 0.9, 0.05),
    (4200, 3, 1, 264, 1056, 0.3, 0.0),
    (64, 8, 2, 136, 256, 0.0, 1.0),                            # nobody has an expert
]


@pytest.mark.parametrize("T,E,k,N,K,skew,missing", CASES)
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
def test_product(metis, T, E, k, N, K, skew, missing, gather, dtype, out):
    plan, g = _plan(metis, T, E, k, T + N, skew, missing)
    x, w = _dense(g, T if gather else T * k, K, dtype), _dense(g, E * N, K, torch.bfloat16)
    W = metis.MxTensor(E * N, K)
    metis.quantize_mx(w.cuda(), W)
    offsets, token = plan.offsets.cpu().numpy(), plan.token.cpu().numpy()
    ref = oe.experts_product(x.double().numpy(), _codes(W), offsets, token, gather)
    wq = omx.dequantize_mx(*_codes(W))
    big = oe.experts_product(x.double().abs().numpy(), omx.quantize_mx(np.abs(wq)), offsets, token, gather)
    for pad in (0, 5):
        xd = torch.zeros((x.shape[0], K + 8 * pad), dtype=dtype, device="cuda")
        xd[:, 8 * pad:] = x.cuda()
        C = torch.full((T * k, N + pad), float("nan"), dtype=out, device="cuda")
        metis.experts_product(xd[:, 8 * pad:], W, plan, C[:, pad:], gather=gather)
        _check(C[:, pad:], ref, big, out)
        assert torch.isnan(C[:, :pad]).all()
    assert not C[int(offsets[-1]):, 5:].any()


def test_product_is_the_dense_one_where_there_is_one_expert(metis):
    """One expert, every token once: the same bits as metis_mxfp4_gemm_nt of the same operands."""
    T, N, K = 777, 640, 1024
    g = torch.Generator().manual_seed(0)
    plan = metis.dispatch(torch.zeros((T, 1), dtype=torch.int32, device="cuda"), 1)
    x, w = _dense(g, T, K, torch.bfloat16).cuda(), _dense(g, N, K, torch.bfloat16).cuda()
    X, W = metis.MxTensor(T, K), metis.MxTensor(N, K)
    metis.quantize_mx(x, X)
    metis.quantize_mx(w, W)
    want = metis.mxfp4_gemm_nt(X, W, torch.empty((T, N), device="cuda"))
    got = metis.experts_product(x, W, plan, torch.empty((T, N), device="cuda"), gather=True)
    assert float((got - want).abs().max()) <= 2e-6 * float(want.abs().max()) * 16


@pytest.mark.parametrize("groups,M,N", [(1, 32, 8), (3, 96, 72), (2, 512, 264), (5, 64, 1024)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_mx_t_bit_exact(metis, groups, M, N, dtype):
    g = torch.Generator().manual_seed(M + N)
    x = _dense(g, groups * M, N, dtype, 2.0)
    x[:8, 0] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    x[8:32, 0] = 0.0
    x[9, 0] = 7.5
    x[:32, 1] = 0.0
    x[3, 1] = -0.0
    x[:32, 2] = 2.0 ** -130
    wide = torch.zeros((groups * M, N + 16), dtype=dtype, device="cuda")
    wide[:, 8:8 + N] = x.cuda()
    for xd in (x.cuda(), wide[:, 8:8 + N]):
        q = metis.MxTensor(groups * N, M)
        q.codes.fill_(0xA5)
        q.scales.fill_(0xA5)
        metis.quantize_mx_t(xd, q, groups)
        c, s = omx.quantize_mx(x.double().numpy().reshape(groups, M, N).transpose(0, 2, 1).reshape(groups * N, M))
        assert np.array_equal(_codes(q)[1], s) and np.array_equal(_codes(q)[0], c)


@pytest.mark.parametrize("T,E,k,N,K,skew,missing", [c if c[3] % 8 == 0 else c[:3] + (c[3] // 8 * 8 + 8,) + c[4:] for c in CASES])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
def test_weight_gradient(metis, T, E, k, N, K, skew, missing, gather, dtype, out):
    plan, g = _plan(metis, T, E, k, T + N, skew, missing)
    x, dy = _dense(g, T if gather else T * k, K, dtype), _dense(g, T * k, N, dtype)
    offsets, token = plan.offsets.cpu().numpy(), plan.token.cpu().numpy()
    dy[int(offsets[-1]):] = float("nan")                       # unused slots are not read
    xn, dn = x.double().numpy(), dy.double().nan_to_num(0.0).numpy()
    ref = oe.experts_wgrad(dn, xn, offsets, token, gather)
    big = oe.experts_wgrad(np.abs(dn), np.abs(xn), offsets, token, gather)
    for pad in (0, 3):
        dW = torch.full((E * N, K + pad), float("nan"), dtype=out, device="cuda")
        metis.experts_wgrad(dy.cuda(), x.cuda(), plan, dW[:, pad:], gather=gather)
        _check(dW[:, pad:], ref, big, out)
        assert torch.isnan(dW[:, :pad]).all()


@pytest.mark.parametrize("T", [40, 900])
@pytest.mark.parametrize("gt,xt", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_weight_gradient_of_two_types(metis, T, gt, xt):
    E, k, N, K = 5, 2, 136, 328
    plan, g = _plan(metis, T, E, k, T, 0.3, 0.1)
    x, dy = _dense(g, T, K, xt), _dense(g, T * k, N, gt)
    offsets, token = plan.offsets.cpu().numpy(), plan.token.cpu().numpy()
    ref = oe.experts_wgrad(dy.double().numpy(), x.double().numpy(), offsets, token, True)
    big = oe.experts_wgrad(dy.double().abs().numpy(), x.double().abs().numpy(), offsets, token, True)
    dW = torch.full((E * N, K), float("nan"), device="cuda")
    metis.experts_wgrad(dy.cuda(), x.cuda(), plan, dW, gather=True)
    _check(dW, ref, big, torch.float32)


def test_no_tokens(metis):
    plan = metis.dispatch(torch.empty((0, 2), dtype=torch.int32, device="cuda"), 8)
    e = lambda n: torch.empty((0, n), dtype=torch.bfloat16, device="cuda")
    W = metis.MxTensor(8 * 16, 64)
    metis.experts_product(e(64), W, plan, e(16))
    dW = torch.full((8 * 16, 64), 3.0, device="cuda")
    metis.experts_wgrad(e(16), e(64), plan, dW)
    assert not dW.any()


def test_on_another_stream_and_in_a_graph(metis):
    T, E, k, N, K = 300, 8, 2, 256, 512
    plan, g = _plan(metis, T, E, k, 1, 0.5, 0.1)
    x, dy, w = _dense(g, T, K, torch.bfloat16).cuda(), _dense(g, T * k, N, torch.bfloat16).cuda(), _dense(g, E * N, K, torch.bfloat16).cuda()
    W = metis.MxTensor(E * N, K)
    metis.quantize_mx(w, W)
    C0 = metis.experts_product(x, W, plan, torch.empty((T * k, N), dtype=torch.bfloat16, device="cuda"), gather=True)
    dW0 = metis.experts_wgrad(dy, x, plan, torch.empty((E * N, K), device="cuda"), gather=True)
    C1, dW1 = torch.empty_like(C0), torch.empty_like(dW0)
    ws = torch.empty((max(metis.experts_workspace_bytes(T, T * k, E, N, K), metis.experts_wgrad_workspace_bytes(T * k, E, N, K)),), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        metis.experts_product(x, W, plan, C1, gather=True, workspace=ws)
        metis.experts_wgrad(dy, x, plan, dW1, gather=True, workspace=ws)
    for _ in range(3):
        C1.fill_(float("nan"))
        dW1.fill_(float("nan"))
        ws.random_(0, 256)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(C0, C1) and torch.equal(dW0, dW1)
