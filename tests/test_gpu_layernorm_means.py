"""Layer norm of rows whose spread is small beside their mean, as small as the last place of the mean itself.

u = 2^-24.  The row's sum is held in 64 bits: the mean is off by at most n 2^-53 mean|x|, and by 2 u^2 |mean| as two fp32 numbers (e0, together).  Eight
bf16 elements are summed in fp32 first, which is exact unless they are more than 2^13 times apart: up to 7 u mean|x| more in such rows.  A difference to
the mean rounds twice, so it is off by 2 u |d| + e0.  The variance sums at most 64 u and three roundings of each term: relatively, with the differences'
errors, 74 u + 2 e0 rstd + (e0 rstd)^2; rstd is off by half of that and four roundings.  Results round once more: 2^-8 for bf16, u for fp32."""
import numpy as np
import pytest
import torch

from oracle import epilogue as oep

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float32: u}
WIDTHS = [1, 5, 8, 64, 300, 1000, 2048, 4096, 5000, 8192, 16384, 16390, 50000]


@pytest.fixture(scope="module")
def metis():
    from paper_2509_00404_amd import metis as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def _f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_equal_elements(metis, D, dtype):
    values = torch.tensor([0.1, 1000.3, 12345.678, -7.7, 1e-30, 2.9e38]).to(dtype)
    x = values[:, None].repeat(1, D).cuda()
    stats = torch.empty((len(values), 2), device="cuda")
    y = metis.layernorm(x, torch.empty_like(x), None, None, 1e-5, stats)
    assert (y == 0).all() and torch.equal(stats[:, 0].cpu(), values.float())
    assert ((stats[:, 1].cpu().double() / float(np.float32(1e-5)) ** -0.5 - 1).abs() <= 4 * u).all()
    w, b = torch.randn(D, device="cuda"), torch.randn(D, device="cuda")
    assert torch.equal(metis.layernorm(x, torch.empty_like(x), w, b), b.to(dtype).expand_as(x))
    assert torch.isnan(metis.layernorm(x, torch.empty_like(x), w, b, 0.0)).all()


def _rows(D, dtype, seed):
    """Rows of mean c whose elements are a few last places of c apart, rows with a single element off by one, and rows far from zero with unit spread."""
    g = torch.Generator().manual_seed(seed)
    rows = []
    for c in (0.1, 1000.3, -12345.678):
        c = torch.tensor(c).to(dtype)
        place = 2.0 ** (np.floor(np.log2(abs(c.item()))) - (7 if dtype == torch.bfloat16 else 23))
        rows.append(c.double() + place * torch.randint(-8, 9, (D,), generator=g))
        one = torch.full((D,), c.item(), dtype=torch.float64)
        one[D // 3] += place
        rows.append(one)
        rows.append((c.double() + torch.randn(D, generator=g)))
    rows.append(torch.randn(D, generator=g).double())
    rows[-1][D // 2] = 1e4
    return torch.stack(rows).to(dtype)


@pytest.mark.parametrize("D", [d for d in WIDTHS if d >= 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_rows_of_little_spread(metis, D, dtype, eps):
    x = _rows(D, dtype, D)
    w, b = 1 + 0.3 * torch.randn(D, generator=torch.Generator().manual_seed(1)), 0.1 * torch.randn(D, generator=torch.Generator().manual_seed(2))
    x64, eps64 = _f64(x), np.float32(eps).astype(np.float64)
    x64 = x64.astype(np.longdouble)                                  # (the reference's own mean would be off by as much as e0)
    mean = x64.mean(1, keepdims=True)
    d = (x64 - mean).astype(np.float64)
    if eps == 0.0:                                                   # rows of equal elements (bf16's unit spread is below its last place there) have no rstd
        some = np.any(d != 0, 1)
        y = metis.layernorm(x.cuda(), torch.empty_like(x, device="cuda"), eps=eps).cpu()
        assert torch.isnan(y[torch.from_numpy(~some)]).all() and some.sum() >= 8
        x, x64, mean, d = x[torch.from_numpy(some)], x64[some], mean[some], d[some]
    rstd = 1 / np.sqrt((d * d).mean(1, keepdims=True) + eps64)
    xh = d * rstd
    mean = mean.astype(np.float64)
    e0 = D * 2.0 ** -53 * np.abs(x64).mean(1, keepdims=True).astype(np.float64) + 2 * u * u * np.abs(mean)
    if dtype == torch.bfloat16:
        size = np.abs(_f64(x))
        apart = size.max(1, keepdims=True) > 2.0 ** 13 * size.min(1, keepdims=True)
        e0 = e0 + np.where(apart, 7 * u * size.mean(1, keepdims=True), 0.0)
    er = 0.5 * (74 * u + 2 * e0 * rstd + (e0 * rstd) ** 2) + 4 * u
    for weight, bias in ((None, None), (w, b)):
        stats = torch.empty((len(x), 2), device="cuda")
        y = metis.layernorm(x.cuda(), torch.empty_like(x, device="cuda"), weight.cuda() if weight is not None else None,
                            bias.cuda() if bias is not None else None, eps, stats)
        ww, bb = (1.0, 0.0) if weight is None else (_f64(weight), _f64(bias))
        ref = xh * ww + bb
        err = np.abs(ww) * (np.abs(xh) * (er + 4 * u) + rstd * (2 * u * np.abs(d) + e0) * (1 + er)) + 2 * u * np.abs(ref) + u * np.abs(bb)
        off = np.abs(_f64(y) - ref) - err - ROUND[dtype] * (np.abs(ref) + err)
        assert np.all(off <= 0), (off.max(1), np.abs(xh).max(1))
        s = _f64(stats)
        assert np.all(np.abs(s[:, :1] - mean) <= u * np.abs(mean) + e0) and np.all(np.abs(s[:, 1:] / rstd - 1) <= er)


def test_sums_beyond_fp32(metis):
    """Elements whose sum passes fp32's range, and whose mean does not."""
    for D in (300, 4096, 16390):
        x = torch.full((2, D), 3e38, device="cuda")
        x[1, ::2] = -3e38
        stats = torch.empty((2, 2), device="cuda")
        y = metis.layernorm(x, torch.empty_like(x), stats=stats)
        assert (y[0] == 0).all() and stats[0, 0] == x[0, 0] and torch.isfinite(stats[1, 0])
