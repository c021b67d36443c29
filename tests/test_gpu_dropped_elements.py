"""A dropped element has no part in the backward pass, whatever the forward pass left there: NaN and infinities in its place change no bit of dz and dbias."""
import functools

import numpy as np
import pytest
import torch

from oracle import epilogue as oep

pytestmark = pytest.mark.gpu
BAD = torch.tensor([float("nan"), float("inf"), float("-inf")])


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


@functools.lru_cache(maxsize=1)
def _dropped(T, N):
    return torch.from_numpy(oep.mask(0.3, 21, 0, np.arange(T), N) == 0).cuda()


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,N", [(3, 9), (2, 5), (40, 2057), (768, 64), (900, 77), (900, 512), (800, 2057), (800, 4096), (32768, 2048)])
def test_gradient(metis, T, N, dtype, act):
    g = torch.Generator().manual_seed(T + N)
    dy, pre = (torch.randn((T, N), generator=g).to(dtype).cuda() for _ in range(2))
    mask = metis.DropoutMask(0.3, 21)
    dropped = _dropped(T, N)
    assert dropped.any() and not dropped.all()
    bad = BAD.cuda().to(dtype)[torch.randint(0, 3, (T, N), generator=g).cuda()]
    db = [torch.empty(N, device="cuda") for _ in range(3)]
    dz = [metis.linear_grads(dy, torch.empty_like(dy), pre=pre, act=act, mask=mask, dbias=db[0])]
    dz.append(metis.linear_grads(dy, torch.empty_like(dy), pre=torch.where(dropped, bad, pre), act=act, mask=mask, dbias=db[1]))
    dz.append(metis.linear_grads(torch.where(dropped, bad, dy), torch.empty_like(dy), pre=torch.where(dropped, bad, pre), act=act, mask=mask, dbias=db[2]))
    assert (dz[0][dropped] == 0).all() and torch.isfinite(dz[0]).all() and torch.isfinite(db[0]).all()
    for z, s in zip(dz[1:], db[1:]):
        assert torch.equal(z, dz[0]) and torch.equal(s, db[0])


@pytest.mark.parametrize("T,N", [(5, 40), (900, 77), (800, 4096)])
def test_kept_elements_keep_their_missing_values(metis, T, N):
    dy, pre, db = torch.ones((T, N), device="cuda"), torch.zeros((T, N), device="cuda"), torch.empty(N, device="cuda")
    kept = oep.mask(0.3, 21, 0, [1], N)[0] > 0
    at = int(np.argmax(kept))
    pre[1, at] = float("nan")
    for act in ("relu", "gelu", "gelu_tanh", "silu"):
        dz = metis.linear_grads(dy, torch.empty_like(dy), pre=pre, act=act, mask=metis.DropoutMask(0.3, 21), dbias=db)
        assert torch.isnan(dz).sum() == 1 and torch.isnan(dz[1, at]) and torch.isnan(db).sum() == 1 and torch.isnan(db[at])
