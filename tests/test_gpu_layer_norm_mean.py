"""Layer norm of rows whose mean is large against their spread."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# rows of lanes of a wave, of a wave, of whole waves (many rows, few rows), past the registers; odd ends
SIZES = ((20000, 7), (5000, 64), (300, 1000), (3000, 1500), (3000, 4096), (40, 4096), (40, 12289), (9, 70000))


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("mean,spread", [(1e4, 1.0), (-3e5, 2.0), (1000.0, 1.5)])
def test_deviations_do_not_carry_the_rounding_of_the_mean(size, mean, spread):
    rows, c = size
    gen = torch.Generator().manual_seed(c)
    x = (mean + spread * torch.randn(rows, c, generator=gen, dtype=torch.float64)).float()
    y, m, r = scnn.layer_norm_fwd(x.to(DEV), eps=1e-5)
    v = x.double()
    exact = v.mean(1, keepdim=True)
    d = v - exact
    rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5)
    # squares: 64 + c / 1024 roundings of a sum of fp32, of which the root takes half; difference, difference, product, root,
    # quotient, product; the mean itself is good to fp64's roundings
    rel = (0.5 * (64 + c / 1024) + 8) * ref.U32
    slip = 8 * 2.0 ** -53 * v.abs().amax(1, keepdim=True) * rstd
    ref.assert_within(y, (d * rstd, rel * (d * rstd).abs() + slip + ref.tiny(torch.float32)), "out")
    ref.assert_within(r, (rstd[:, 0], (rel * rstd)[:, 0]), "rstd")
    ref.assert_within(m, (exact[:, 0], (1 + 1e-6) * ref.U32 * exact.abs()[:, 0]), "mean")  # rounded once


@pytest.mark.parametrize("channels", [7, 25, 1000, 12289, 70000])
def test_rows_of_equal_values_have_no_deviations(channels):
    values = torch.tensor([1e30, -3.3e38, 0.1, 1 / 3, 7e-39, 12345.678, 0.0])
    x = values[:, None].expand(-1, channels).contiguous().to(DEV)
    beta = torch.randn(channels, generator=torch.Generator().manual_seed(1)).to(DEV)
    y, m, _ = scnn.layer_norm_fwd(x, None, beta)
    assert torch.equal(y, beta.expand(len(values), -1)) and torch.equal(m.cpu(), values)


def test_a_row_with_an_infinity():
    x = torch.randn(4, 300, generator=torch.Generator().manual_seed(2)).to(DEV)
    x[1, 7] = float("inf")
    x[2, 9] = -float("inf")
    y, m, r = scnn.layer_norm_fwd(x)
    assert torch.isnan(y[1:3]).all() and torch.isfinite(y[::3]).all()
    assert float(m[1]) == float("inf") and float(m[2]) == -float("inf") and torch.isnan(r[1:3]).all()
