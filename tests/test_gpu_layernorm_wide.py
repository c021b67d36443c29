"""Layer norm at the widest rows it takes, and its gradients: the columns' sums of all columns."""
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


@pytest.mark.parametrize("N", [(1 << 27) + 5, 1 << 28])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_row(metis, N, dtype):
    """Equal elements are 0 exactly; of two values beside each other, d apart and in turn, the mean is between them and the results are +-1.  The sum is
    exact (whole multiples of 2^-14 below 2^38: 52 bits), the mean 1 / N off the middle where N is odd, the variance within 2^-16 (sums of eight terms in fp32,
    the rest in 64 bits), and the results round once more."""
    x = torch.full((1, N), 1000.3, device="cuda").to(dtype)
    stats = torch.empty((1, 2), device="cuda")
    y = metis.layernorm(x, torch.empty_like(x), stats=stats)
    assert (y == 0).all() and stats[0, 0] == x[0, 0].float()
    d = 4.0 if dtype == torch.bfloat16 else 2.0 ** -13
    x[0, 1::2] += d
    y = metis.layernorm(x, torch.empty_like(x), eps=0.0, stats=stats)
    off = 4.0 / N + 2.0 ** -16
    last = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    assert (y[0, 0::2].float() + 1).abs().max() <= off + last and (y[0, 1::2].float() - 1).abs().max() <= off + last
    assert abs(stats[0, 1].item() * d / 2 - 1) <= off
