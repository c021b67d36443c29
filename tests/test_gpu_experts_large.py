"""The mixture-of-experts calls where one workgroup has many tiles, and where offsets pass 32 bits: the far end of a large operand gives what
the same rows give by themselves."""
import numpy as np
import pytest
import torch

from oracle import experts as oe
from test_gpu_experts import _check, _codes, _dense, _plan

from oracle import mx as omx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("T,E,k,N,K,skew", [(3000, 6, 2, 4200, 288, 0.3), (2600, 60, 4, 1100, 512, 0.0)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_product_over_many_tiles(metis, T, E, k, N, K, skew, out):
    plan, g = _plan(metis, T, E, k, 11, skew, 0.05)
    x, w = _dense(g, T, K, torch.bfloat16), _dense(g, E * N, K, torch.bfloat16)
    W = metis.MxTensor(E * N, K)
    metis.quantize_mx(w.cuda(), W)
    offsets, token = plan.offsets.cpu().numpy(), plan.token.cpu().numpy()
    ref = oe.experts_product(x.double().numpy(), _codes(W), offsets, token, True)
    big = oe.experts_product(x.double().abs().numpy(), omx.quantize_mx(np.abs(omx.dequantize_mx(*_codes(W)))), offsets, token, True)
    C = torch.full((T * k, N), float("nan"), dtype=out, device="cuda")
    metis.experts_product(x.cuda(), W, plan, C, gather=True)
    _check(C, ref, big, out)


@pytest.mark.parametrize("T,E,k,N,K,skew", [(1500, 6, 2, 2312, 3000, 0.3), (700, 20, 4, 1032, 1800, 0.0),
                                               (300, 40, 4, 1096, 1160, 0.5)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_weight_gradient_over_many_tiles(metis, T, E, k, N, K, skew, out):
    plan, g = _plan(metis, T, E, k, 12, skew, 0.05)
    x, dy = _dense(g, T, K, torch.bfloat16), _dense(g, T * k, N, torch.bfloat16)
    offsets, token = plan.offsets.cpu().numpy(), plan.token.cpu().numpy()
    ref = oe.experts_wgrad(dy.double().numpy(), x.double().numpy(), offsets, token, True)
    big = oe.experts_wgrad(dy.double().abs().numpy(), x.double().abs().numpy(), offsets, token, True)
    dW = torch.full((E * N, K), float("nan"), dtype=out, device="cuda")
    metis.experts_wgrad(dy.cuda(), x.cuda(), plan, dW, gather=True)
    _check(dW, ref, big, out)


@pytest.mark.parametrize("T", [5, 1100])                       # straight from memory, and the stream
def test_weights_past_32_bits(metis, T):
    E, N, K = 66, 16384, 8192                                  # 4.4 GB of codes
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 256, (E * N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(118, 124, (E * N, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    W = metis.MxTensor(E * N, K, buffers=(codes, scales))
    last = metis.MxTensor(N, K, buffers=(codes[-N:].contiguous(), scales[-N:].contiguous()))
    x = torch.randn((T, K), generator=g, device="cuda").to(torch.bfloat16)
    plan = metis.dispatch(torch.full((T, 1), E - 1, dtype=torch.int32, device="cuda"), E)
    got = metis.experts_product(x, W, plan, torch.empty((T, N), device="cuda"), gather=True)
    X = metis.quantize_mx(x, metis.MxTensor(T, K))
    want = metis.mxfp4_gemm_nt(X, last, torch.empty((T, N), device="cuda"))
    assert float((got - want).abs().max()) <= 1e-5 * float(want.abs().max())


def test_rows_past_32_bits(metis):
    T, k, D = 150000, 4, 4096                                  # 2.4e9 elements
    plan = metis.dispatch(torch.arange(T * k, device="cuda", dtype=torch.int32).view(T, k) % 8, 8)
    rows = torch.empty((T * k, D), dtype=torch.bfloat16, device="cuda")
    rows.copy_((torch.arange(T * k, device="cuda") % 251 - 125)[:, None] * (torch.arange(D, device="cuda") % 13 + 1))
    w = torch.rand((T, k), device="cuda")
    y = metis.combine(rows, plan, torch.empty((T, D), dtype=torch.bfloat16, device="cuda"), w)
    t = torch.tensor([0, T // 2, T - 1], device="cuda")
    slot = plan.slot[t].long()
    want = (rows[slot].double() * w[t].double()[..., None]).sum(1)
    assert int(slot.max()) * D > 2 ** 31
    big = (rows[slot].double().abs() * w[t].double()[..., None]).sum(1)
    assert bool(((y[t].double() - want).abs() <= 2.0 ** -8 * big).all())
    dy = y
    drows, dw = metis.combine_grads(dy, rows, plan, w)
    want = dy[t].double()[:, None] * w[t].double()[..., None]
    assert bool(((drows[slot].double() - want).abs() <= 1.01 * 2.0 ** -8 * want.abs()).all())
    want = (dy[t].double()[:, None] * rows[slot].double()).sum(2)
    big = (dy[t].double()[:, None] * rows[slot].double()).abs().sum(2)
    assert bool(((dw[t].double() - want).abs() <= 2e-5 * big).all())


def test_checkpoints_past_32_bits(metis):
    S, F = 1100000, 1024                                       # 2.25e9 codes, 4.5 GB of bf16
    gu = torch.empty((S, 2 * F), dtype=torch.bfloat16, device="cuda").normal_()
    act, q = torch.empty((S, F), dtype=torch.bfloat16, device="cuda"), metis.Mx8Tensor(S, 2 * F)
    metis.swiglu(gu, act, q)
    dgu, again = torch.empty_like(gu), torch.empty_like(act)
    metis.swiglu_grads(q, act, dgu, again)
    n = 5
    tail = gu[-n:].contiguous()
    act1, q1 = torch.empty((n, F), dtype=torch.bfloat16, device="cuda"), metis.Mx8Tensor(n, 2 * F)
    metis.swiglu(tail, act1, q1)
    dgu1, again1 = torch.empty_like(tail), torch.empty_like(act1)
    metis.swiglu_grads(q1, act1, dgu1, again1)
    assert torch.equal(act[-n:], act1) and torch.equal(q.codes[-n:], q1.codes) and torch.equal(q.scales[-n:], q1.scales)
    assert torch.equal(dgu[-n:], dgu1) and torch.equal(again[-n:], again1)
    back = metis.dequantize_mx8(q, dgu)
    assert torch.equal(back[-n:], metis.dequantize_mx8(q1, dgu1))


def _values(codes, scales):
    """fp64 values of MXFP4 rows on the GPU"""
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
    v = grid[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (v.unflatten(-1, (-1, 32)) * torch.exp2(scales.double() - 127)[..., None]).flatten(-2)


def test_product_over_more_tiles_than_are_looked_up_at_once(metis):
    T, E, N, K = 1100, 64, 98304, 64                           # about a hundred tiles a workgroup
    g = torch.Generator(device="cuda").manual_seed(3)
    codes = torch.randint(0, 256, (E * N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(120, 126, (E * N, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    W = metis.MxTensor(E * N, K, buffers=(codes, scales))
    x = torch.randn((T, K), generator=g, device="cuda").to(torch.bfloat16)
    idx = torch.randint(0, E, (T, 1), generator=g, device="cuda", dtype=torch.int32)
    plan = metis.dispatch(idx, E)
    C = torch.full((T, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    metis.experts_product(x, W, plan, C, gather=True)
    X = metis.quantize_mx(x, metis.MxTensor(T, K))
    xv = _values(X.codes, X.scales)[plan.token.long()]
    expert = idx[plan.token.long(), 0].long()
    cols = torch.cat((torch.arange(600, device="cuda"), torch.randint(0, N, (600,), generator=g, device="cuda"), torch.arange(N - 600, N, device="cuda")))
    assert bool(torch.isfinite(C).all())
    for e in range(E):
        s = (expert == e).nonzero()[:, 0]
        wv = _values(codes[e * N + cols], scales[e * N + cols])
        ref, big = xv[s] @ wv.T, xv[s].abs() @ wv.abs().T
        assert bool(((C[s][:, cols].double() - ref).abs() <= 2e-6 * big + 2.0 ** -8 * ref.abs()).all()), e


def test_weight_gradient_over_more_tiles_than_are_looked_up_at_once(metis):
    T, E, N, K = 300, 2, 28416, 28672
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.randn((T, n), generator=g, device="cuda").to(torch.bfloat16) for n in (K, N))
    plan = metis.dispatch((torch.rand((T, 1), generator=g, device="cuda") < 0.4).to(torch.int32), E)
    dW = torch.full((E * N, K), float("nan"), dtype=torch.bfloat16, device="cuda")
    metis.experts_wgrad(dy, x, plan, dW, gather=True)
    ends = plan.offsets.tolist()
    assert min(ends[1], T - ends[1]) > 64
    rows = torch.cat((torch.arange(300, device="cuda"), torch.randint(0, N, (300,), generator=g, device="cuda"), torch.arange(N - 300, N, device="cuda")))
    for e in range(E):
        s = torch.arange(ends[e], ends[e + 1], device="cuda")
        pad = (0, 0, 0, -len(s) % 32)
        q = [torch.nn.functional.pad(t, pad).t().contiguous() for t in (dy[s][:, rows], x[plan.token[s].long()])]
        v = [_values(m.codes, m.scales) for m in (metis.quantize_mx(t, metis.MxTensor(*t.shape)) for t in q)]
        ref, big = v[0] @ v[1].T, v[0].abs() @ v[1].abs().T
        got = dW[e * N + rows].double()
        assert bool(torch.isfinite(got).all()) and bool(((got - ref).abs() <= 2e-6 * big + 2.0 ** -8 * ref.abs()).all()), e
