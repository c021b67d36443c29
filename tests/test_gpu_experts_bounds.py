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


def _offsets_that_descend(S, E, seed):
    """offsets with dips, negative ones and ones behind the slots, and what they are held to: their running maximum within 0 .. S"""
    g = torch.Generator().manual_seed(seed)
    o = torch.sort(torch.randint(0, S + 1, (E + 1,), generator=g)).values
    dip = torch.rand((E + 1,), generator=g) < 0.4
    o[dip] -= torch.randint(1, 2 * S, (int(dip.sum()),), generator=g)
    if seed % 2:
        o[E - E // 8:] = S + 7                                 # the last experts behind the slots
    o[0], o[E // 2], o[E] = -3, -1, S
    held = torch.cummax(o.clamp(0, S), 0).values
    assert bool((o[1:] < o[:-1]).any()) and int(held[0]) == 0
    return o.to(torch.int32).cuda(), held.to(torch.int32).cuda()


@pytest.mark.parametrize("T,E,k,N,K", [
    (3, 8, 4, 72, 256),                                        # a decode step
    (60, 160, 4, 200, 992),                                    # few slots
    (1100, 4, 2, 520, 160),                                    # the stream
    (2200, 130, 2, 264, 320),
    (600, 9, 2, 320, 4096),                                    # the contraction in parts
])
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_offsets_that_do_not_ascend(metis, T, E, k, N, K, seed):
    """Read as their running maximum, within the slots: the bits of the plan that has that, and nothing written elsewhere."""
    S = T * k
    g = torch.Generator(device="cuda").manual_seed(seed)
    token = torch.randint(0, T, (S,), generator=g, device="cuda", dtype=torch.int32)
    slot = torch.randperm(S, generator=g, device="cuda").to(torch.int32).view(T, k)
    x, dy = (torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16) for shape in ((S, K), (S, N)))
    W = metis.quantize_mx(torch.randn((E * N, K), generator=g, device="cuda").to(torch.bfloat16), metis.MxTensor(E * N, K))
    results = []
    for offsets in _offsets_that_descend(S, E, seed):
        plan = metis.ExpertPlan(T, E, k, buffers=(offsets, token, slot))
        C = torch.full((S + 8, N), float("nan"), dtype=torch.bfloat16, device="cuda")
        ws, end = _guarded(metis.experts_workspace_bytes(S, S, E, N, K), 1 << 20)
        metis.experts_product(x, W, plan, C[:S], workspace=ws)
        assert bool(torch.isnan(C[S:]).all()) and bool((end == 0xA5).all())
        out = [C[:S]]
        for dtype in (torch.bfloat16, torch.float32):
            dW = torch.full((E * N + 8, K), float("nan"), dtype=dtype, device="cuda")
            ws, end = _guarded(metis.experts_wgrad_workspace_bytes(S, E, N, K), 1 << 20)
            metis.experts_wgrad(dy, x, plan, dW[:E * N], workspace=ws)
            assert bool(torch.isnan(dW[E * N:]).all()) and bool((end == 0xA5).all())
            out.append(dW[:E * N])
        results.append(out)
    for got, want in zip(*results):
        assert bool(torch.isfinite(want).all()) and torch.equal(got, want)
