"""GPU parity of the routing to experts with the fp64 oracle: selection, weights, gradient, plan.

Logits of the selection tests are multiples of 1/8, so that many tie and no two others are near each other: softmax keys (x + bias, bias a multiple of
1/8) are exact, and distinct sigmoid keys here are checked to be apart by more than fp32's rounding.  Weights: an exponential and a
quotient of a few ulp each, sums over at most 512 terms -> 1e-5 relative to the row's largest; gradients the same relative to the largest in the row."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import experts as oe

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def _logits(T, E, seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = torch.round(8 * 1.5 * torch.randn((T, E), generator=g)) / 8
    if T > 8 and E > 4:
        x[1] = -np.inf                                        # no expert at all
        x[2, 1:] = -np.inf                                    # a single one
        x[3, 1:] = torch.finfo(dtype).min                     # masked by the type's lowest value: available, weight 0
        x[4, ::2] = float("nan")
        x[5] = 0.25                                           # all tie
        x[6, :3] = torch.tensor([0.0, -0.0, 0.0])
        x[7] = -88.0                                          # scores near the end of the range
        x[8] = -torch.arange(E) * 200.0
    return x.to(dtype)


def _close_rows(got, ref, tol):
    big = np.abs(ref).max(axis=1, keepdims=True)
    assert np.all(np.isfinite(got))
    assert np.max(np.abs(got - ref) / np.where(big > 0, big, 1.0)) < tol


@pytest.mark.parametrize("T,E,k,groups,top_groups", [(1, 64, 4, 1, 1), (33, 8, 2, 1, 1), (100, 60, 6, 4, 2), (257, 256, 8, 8, 4), (64, 5, 5, 1, 1),
                                                     (40, 512, 16, 16, 3), (17, 1, 1, 1, 1), (50, 12, 3, 12, 5), (31, 160, 6, 5, 1)])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_route(metis, T, E, k, groups, top_groups, scores, renorm):
    x = _logits(T, E, T + E)
    g = torch.Generator().manual_seed(T)
    for biased in (False, True):
        bias = torch.round(8 * torch.randn((E,), generator=g)) / 8 if biased else None
        valid = (torch.rand((T,), generator=g) > 0.2).to(torch.uint8) if biased else None
        if biased and E > 8:
            bias[3] = -np.inf
        idx, w = metis.route(x.cuda(), k, bias=None if bias is None else bias.cuda(), valid=None if valid is None else valid.cuda(),
                             scores=scores, groups=groups, top_groups=top_groups, renorm=renorm, scale=2.5)
        ri, rw = oe.route(x.double().numpy(), k, None if bias is None else bias.double().numpy(), None if valid is None else valid.numpy(),
                          scores, groups, top_groups, renorm, 2.5)
        torch.cuda.synchronize()
        same = np.ones(T, dtype=bool)
        if scores == "sigmoid":                               # rows whose distinct keys (or group scores) are nearer than fp32 tells apart
            for t in range(T):
                key = oe.selection_keys(x[t].double().numpy(), None if bias is None else bias.double().numpy(), scores)
                vals = np.concatenate([key, oe.group_scores(key, groups, scores)])
                gap = np.diff(np.unique(vals[vals > -np.inf]))
                same[t] = not np.any(gap < 1e-6)
            assert same.mean() > 0.5
        assert np.array_equal(idx.cpu().numpy()[same], ri[same])
        _close_rows(w.double().cpu().numpy()[same], rw[same], 1e-5)


@pytest.mark.parametrize("T,E,k,groups,top_groups", [(65, 256, 8, 8, 4), (40, 512, 16, 16, 3), (33, 128, 4, 1, 1), (20, 384, 5, 3, 2), (9, 248, 6, 1, 1)])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_route_bf16_wide(metis, T, E, k, groups, top_groups, scores):
    """Many experts in bf16: whole 16-byte loads where the rows allow them, single ones in a view off 16 bytes."""
    x = _logits(T, E, E, torch.bfloat16)
    bias = (0.0625 * torch.arange(E) % 1.0)
    ri, rw = oe.route(x.double().numpy(), k, bias.double().numpy(), None, scores, groups, top_groups)
    same = np.ones(T, dtype=bool)
    for t in range(T):
        key = oe.selection_keys(x[t].double().numpy(), bias.double().numpy(), scores)
        vals = np.concatenate([key, oe.group_scores(key, groups, scores)])
        gap = np.diff(np.unique(vals[vals > -np.inf]))
        same[t] = scores == "softmax" or not np.any(gap < 1e-6)
    assert same.mean() > 0.3
    wide = torch.zeros((T, E + 8), dtype=torch.bfloat16, device="cuda")
    for left in (0, 3):
        wide[:, left:left + E] = x.cuda()
        for xd in (x.cuda(), wide[:, left:left + E]):
            idx, w = metis.route(xd, k, bias=bias.cuda(), scores=scores, groups=groups, top_groups=top_groups)
            assert np.array_equal(idx.cpu().numpy()[same], ri[same])
            _close_rows(w.double().cpu().numpy()[same], rw[same], 1e-5)


def test_route_bf16_strided_logits(metis):
    T, E, k = 70, 24, 3
    x = _logits(T, E, 3, torch.bfloat16)
    wide = torch.full((T, E + 7), 100.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:2 + E] = x.cuda()
    idx, w = metis.route(wide[:, 2:2 + E], k)
    ri, rw = oe.route(x.double().numpy(), k)
    assert np.array_equal(idx.cpu().numpy(), ri)
    _close_rows(w.double().cpu().numpy(), rw, 1e-5)


@pytest.mark.parametrize("T,E,k", [(1, 64, 4), (45, 8, 2), (130, 60, 6), (67, 512, 16), (19, 256, 8), (23, 1, 1)])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_grads(metis, T, E, k, scores, renorm):
    g = torch.Generator().manual_seed(E + T)
    x = 1.5 * torch.randn((T, E), generator=g)
    if T > 8 and E > 4:
        x[2, 1:4] = -np.inf
    idx, _ = oe.route(x.double().numpy(), k)
    if T > 8:
        idx[1] = -1                                           # a padding token
        idx[5, 0] = E + 3                                     # outside: no choice
        if k > 1:
            idx[6, 1] = idx[6, 0]                             # listed twice: both count
    dw = torch.randn((T, k), generator=g)
    for dtype, out, tol in ((torch.float32, torch.float32, 1e-5), (torch.bfloat16, torch.bfloat16, 2.0 ** -8), (torch.bfloat16, torch.float32, 1e-5)):
        xd = x.to(dtype)
        ref = oe.route_grads(xd.double().numpy(), idx, dw.double().numpy(), scores, renorm, 0.5)
        got = metis.route_grads(xd.cuda(), torch.from_numpy(idx).to(torch.int32).cuda(), dw.cuda(), scores=scores, renorm=renorm, scale=0.5,
                                out=torch.full((T, E), float("nan"), dtype=out, device="cuda"))
        # the differences in brackets cancel: relative to the largest of v, not of the result
        big = 0.5 * np.abs(dw.double().numpy()).max(axis=1, keepdims=True) * (1.0 if scores == "softmax" or not renorm else 4.0)
        diff = np.abs(got.double().cpu().numpy() - ref)
        assert np.all(np.isfinite(diff)) and np.max(diff / big) < tol


@pytest.mark.parametrize("T,E,k", [(1, 64, 4), (1, 1, 1), (700, 60, 3), (2048, 8, 1), (2049, 512, 16), (16384, 256, 8), (100000, 33, 5)])
@pytest.mark.parametrize("missing", [0.0, 0.1, 1.0])
def test_dispatch(metis, T, E, k, missing):
    rs = np.random.default_rng(T)
    idx = np.minimum(rs.geometric(3.0 / E if E > 3 else 0.9, size=(T, k)) - 1, E - 1)       # few experts have most
    idx[rs.random((T, k)) < missing] = -1
    if T > 1:
        idx[T // 2, 0] = E                                    # outside: no choice
    plan = metis.ExpertPlan(T, E, k)
    for t in (plan.offsets, plan.token, plan.slot):
        t.fill_(-77)
    metis.dispatch(torch.from_numpy(idx).to(torch.int32).cuda(), E, plan)
    flat = idx.reshape(-1)
    there = (flat >= 0) & (flat < E)
    order = np.argsort(np.where(there, flat, E), kind="stable")
    n = there.sum()
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[there], minlength=E))])
    token = np.where(np.arange(T * k) < n, order // k, -1)
    slot = np.full(T * k, -1)
    slot[order[:n]] = np.arange(n)
    if T * k < 5000:                                          # (the oracle's own, one expert at a time)
        ro, rt, rl = oe.plan(np.where((idx >= 0) & (idx < E), idx, -1), E)
        assert np.array_equal(ro, offsets) and np.array_equal(rt, token) and np.array_equal(rl.reshape(-1), slot)
    assert np.array_equal(plan.offsets.cpu().numpy(), offsets)
    assert np.array_equal(plan.token.cpu().numpy(), token)
    assert np.array_equal(plan.slot.cpu().numpy().reshape(-1), slot)


def test_no_tokens(metis):
    idx, w = metis.route(torch.empty((0, 16), device="cuda"), 2)
    plan = metis.dispatch(idx, 16)
    torch.cuda.synchronize()
    assert idx.shape == (0, 2) and plan.offsets.tolist() == [0] * 17
    metis.route_grads(torch.empty((0, 16), device="cuda"), idx, w)


def test_routing_on_another_stream_and_in_a_graph(metis):
    T, E, k = 3000, 64, 4
    x = _logits(T, E, 9).cuda()
    i0, w0 = metis.route(x, k)
    p0 = metis.dispatch(i0, E)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ws = torch.empty((metis.lib().metis_dispatch_workspace_bytes(T, E, k),), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        i1, w1 = metis.route(x, k)
        p1 = metis.dispatch(i1, E, workspace=ws)
    for _ in range(3):
        i1.fill_(-5)
        p1.token.fill_(-5)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(i0, i1) and torch.equal(w0, w1)
        assert torch.equal(p0.token, p1.token) and torch.equal(p0.slot, p1.slot) and torch.equal(p0.offsets, p1.offsets)
