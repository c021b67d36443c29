"""Layer norm's gradients at the widest rows they take: the columns' sums of all columns."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("T,N", [(3, (1 << 26) + 8), (2, 1 << 27), (2, (1 << 27) + 5), (1, 1 << 28)])
def test_sums_of_every_column(metis, T, N):
    """Small whole numbers: the sums are exact."""
    x = (torch.arange(N, device="cuda", dtype=torch.int32) % 251).to(torch.bfloat16).repeat(T, 1)
    dy = torch.ones_like(x)
    dy[0] = 2
    stats = torch.tensor([[1.0, 1.0]], device="cuda").repeat(T, 1)
    dw, db = torch.full((N,), -1.0, device="cuda"), torch.full((N,), -1.0, device="cuda")
    dx = metis.layernorm_grads(dy, x, stats, torch.empty_like(x), dweight=dw, dbias=db)
    assert (db == T + 1).all()
    assert torch.equal(dw, (T + 1) * (x[0].float() - 1))
    assert torch.isfinite(dx).all()
