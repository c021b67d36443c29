"""GPU parity of the experts' rows' way back to the tokens, and of its gradients, with the fp64 oracle.

Sums of k <= 16 terms and of D <= 8192 terms in fp32: an error of at most 2^-24 per term relative to the sum of the terms' magnitudes, 1e-6 for
the short ones and (partial sums of at most D / 256 * 8 terms a lane, then a tree) 2e-5 for the long ones; bf16 results round once more, 2^-8."""
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


def _setup(metis, T, k, D, E, dtype, seed, missing):
    g = torch.Generator().manual_seed(seed)
    idx = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)])
    idx[torch.rand((T, k), generator=g) < missing] = -1
    if T > 3:
        idx[2] = -1                                            # a token without any expert
    plan = metis.dispatch(idx.to(torch.int32).cuda(), E)
    rows = torch.randn((T * k, D), generator=g).to(dtype)
    rows[int(plan.offsets[-1]):] = float("nan")                # unused slots are not read
    w = torch.rand((T, k), generator=g)
    return plan, rows, w, g


CASES = [(1, 4, 64, 8), (5, 1, 8, 4), (33, 4, 1000, 8), (20, 3, 77, 60), (64, 8, 4096, 64), (7, 16, 520, 32), (3, 6, 8192, 16), (40, 2, 1, 4)]


@pytest.mark.parametrize("T,k,D,E", CASES)
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.float32),
                                       (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("missing", [0.0, 0.3])
def test_combine(metis, T, k, D, E, dtype, out, missing):
    plan, rows, w, _ = _setup(metis, T, k, D, E, dtype, T + D, missing)
    slot = plan.slot.cpu().numpy()
    tol = 1e-6 if out == torch.float32 else 2.0 ** -8
    for weights in (w, None):
        for pad in (0, 3):                                     # 3: rows off 16 bytes
            rd = torch.zeros((T * k, D + pad), dtype=dtype, device="cuda")
            rd[:, pad:] = rows.cuda()
            y = torch.full((T, D + pad), 7.0, dtype=out, device="cuda")
            metis.combine(rd[:, pad:], plan, y[:, pad:], None if weights is None else weights.cuda())
            clean = np.nan_to_num(rows.double().numpy())
            ww = None if weights is None else weights.double().numpy()
            ref, big = oe.combine(clean, slot, ww), oe.combine(np.abs(clean), slot, ww)
            assert np.all(np.abs(y[:, pad:].double().cpu().numpy() - ref) <= tol * big)
            assert (y[:, :pad] == 7).all()


@pytest.mark.parametrize("T,k,D,E", CASES)
@pytest.mark.parametrize("dtype,dy_type", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.float32),
                                           (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("missing", [0.0, 0.3])
def test_combine_grads(metis, T, k, D, E, dtype, dy_type, missing):
    plan, rows, w, g = _setup(metis, T, k, D, E, dtype, T + D, missing)
    slot = plan.slot.cpu().numpy()
    dy = torch.randn((T, D), generator=g).to(dy_type)
    clean = np.nan_to_num(rows.double().numpy())
    rdrows, rdw = oe.combine_grads(dy.double().numpy(), clean, slot, w.double().numpy())
    _, big = oe.combine_grads(np.abs(dy.double().numpy()), np.abs(clean), slot, w.double().numpy())
    for pad in (0, 3):
        rd = torch.zeros((T * k, D + pad), dtype=dtype, device="cuda")
        rd[:, pad:] = rows.cuda()
        drows = torch.full((T * k, D + pad), float("nan"), dtype=dtype, device="cuda")
        _, dw = metis.combine_grads(dy.cuda(), rd[:, pad:], plan, w.cuda(), drows=drows[:, pad:])
        got = drows[:, pad:].double().cpu().numpy()
        assert np.all(np.abs(got - rdrows) <= (2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8) * 1.01 * np.abs(rdrows))
        assert torch.isnan(drows[:, :pad]).all()
        assert np.all(np.abs(dw.double().cpu().numpy() - rdw) <= 2e-5 * big)
        again = metis.combine_grads(dy.cuda(), rd[:, pad:], plan, w.cuda())[1]
        assert torch.equal(again, dw)                          # the same bits every time


def test_no_tokens(metis):
    plan = metis.dispatch(torch.empty((0, 2), dtype=torch.int32, device="cuda"), 8)
    e = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    metis.combine(e, plan, e)
    metis.combine_grads(e, e, plan, torch.empty((0, 2), device="cuda"))
