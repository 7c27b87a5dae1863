"""gelu, silu and their slopes where the distribution functions are small, against 64 bits, relative to the value."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rel(z):
    """fp32: a quotient and an exponential good to a last bit (2 U32 each), a fit to 1.3e-7 (2.2) of eight steps whose errors
    shrink with t (3), four products, a fused step: 16 U32 of the value.  The exponential's argument z^2 / 2: the square and its
    product with a constant are rounded, the constant by 0.22 U32, each of the argument: 2.22 U32 z^2 / 2 of the value."""
    return (16 + 1.11 * z * z) * ref.U32


@pytest.mark.parametrize("channels", [24, 4099])  # (from registers; from tiles)
def test_values(channels):
    z = torch.linspace(-12.5, -0.5, channels * 16, dtype=torch.float64).float().view(16, channels)
    one, eye = torch.zeros(16, 1, device=DEV), torch.zeros(1, channels, device=DEV)
    for row in z:
        y, pre = scnn.linear_fwd(one, eye, row.to(DEV), act="gelu", keep_pre=True)
        assert torch.equal(pre.cpu(), row.expand(16, -1))
        want = ref.act(row.double(), "gelu").expand(16, -1)
        ref.assert_within(y, (want, rel(row.double()) * want.abs() + ref.tiny(torch.float32)), "gelu")


@pytest.mark.parametrize("channels", [24, 4099])
def test_slopes(channels):
    z = torch.linspace(-12.5, 3.0, channels * 16, dtype=torch.float64).float().view(16, channels)
    x, w, g = torch.zeros(1, 1, device=DEV), torch.zeros(1, channels, device=DEV), torch.ones(1, channels, device=DEV)
    for row in z:
        _, _, dz = scnn.linear_bwd(x, w, g, act="gelu", pre=row[None].to(DEV))  # (one row: dbias = dz)
        v = row.double()
        cdf = 0.5 * torch.special.erfc(-v / 2 ** 0.5)
        parts = cdf + (ref.act_slope(v, "gelu") - cdf).abs()  # (the slope is their difference below 0)
        ref.assert_within(dz, (ref.act_slope(v, "gelu"), rel(v) * parts + ref.tiny(torch.float32)), "slope")


def test_ends():
    z = torch.tensor([-1e30, -1e10, -64.0, -20.0, 20.0, 1e10, 1e30, 3e38, float("inf"), float("nan")])
    n = len(z)
    y = scnn.linear_fwd(torch.zeros(1, 1, device=DEV), torch.zeros(1, n, device=DEV), z.to(DEV), act="gelu").cpu()[0]
    assert (y[:4] == 0).all() and torch.equal(y[4:9], z[4:9]) and torch.isnan(y[9])
    _, _, dz = scnn.linear_bwd(torch.zeros(1, 1, device=DEV), torch.zeros(1, n, device=DEV), torch.ones(1, n, device=DEV), act="gelu", pre=z[None].to(DEV))
    dz = dz.cpu()
    assert (dz[:4] == 0).all() and (dz[4:8] == 1).all() and torch.isnan(dz[9])


@pytest.mark.parametrize("channels", [24, 4099])
def test_silu(channels):
    # an exponential and a quotient (2 U32 each), a sum, a product; the exponential's argument |z| / ln 2, rounded once and its
    # constant by 0.22 U32; the slope s (1 + z (1 - s)): two sums and two products more, of terms s and |z| s
    z = torch.linspace(-85.0, 3.0, channels * 16, dtype=torch.float64).float().view(16, channels)
    zero, w, g = torch.zeros(1, 1, device=DEV), torch.zeros(1, channels, device=DEV), torch.ones(1, channels, device=DEV)
    for row in z:
        v = row.double()
        off = (6 + 1.22 * v.abs()) * ref.U32
        want = ref.act(v, "silu")[None]
        ref.assert_within(scnn.linear_fwd(zero, w, row.to(DEV), act="silu"), (want, off * want.abs() + ref.tiny(torch.float32)), "silu")
        _, _, dz = scnn.linear_bwd(zero, w, g, act="silu", pre=row[None].to(DEV))
        parts = torch.sigmoid(v) * (1 + v.abs())
        ref.assert_within(dz, (ref.act_slope(v, "silu"), (off + 6 * ref.U32) * parts + ref.tiny(torch.float32)), "slope")
