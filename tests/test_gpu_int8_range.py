"""8-bit linear layers whose rows lie near the ends of fp32's range: the result is finite where the formula's is."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import block_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# one row; 2 to 32 rows, whole and split k; tiles of 64, whole and split k; of 128; of 256
@pytest.mark.parametrize("act", ("none", "relu", "gelu", "silu"))
@pytest.mark.parametrize("rows,c_in,c_out", [(1, 300, 70), (5, 300, 70), (20, 9000, 40), (70, 300, 70), (64, 9000, 70), (3000, 1100, 2900), (8100, 2100, 2043)])
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=str)
def test_large_rows_and_small_weights(dtype, rows, c_in, c_out, act):
    """x up to 3e38 and small w: the sum times the row's scale is past 2^128, times the weight's it is not."""
    gen = torch.Generator().manual_seed(rows)
    x = torch.randn(rows, c_in, generator=gen).clamp(-3, 3)
    x[:, 0] = 3.0
    x[0 if rows == 1 else slice(rows - 1)] *= 1e38
    if rows > 1:  # (and a row of the other end)
        x[-1] *= 2.0 ** -100
    w = torch.randn(c_in, c_out, generator=gen) * (1e-28 * c_in ** -0.5)  # (above 2^-100, the least that a column is held at)
    x, w = x.to(dtype).to(DEV), w.float().to(DEV)
    assert bool(torch.isfinite(x).all())
    q, step = scnn.quantize_weight(w)
    xq, xs = scnn.quantize_rows(x)
    total = xq[:, :c_in].double().cpu() @ q[:, :c_in].double().cpu().t()
    assert bool((total.abs() * xs.double().cpu()[:, None] > 2.0 ** 128).any())
    bias = torch.randn(c_out, generator=gen).to(dtype).to(DEV)
    want = ref.linear_int8(xq, xs, q, step, bias, act, None, dtype)
    assert bool(torch.isfinite(want[0]).all())
    got = scnn.linear_int8_fwd(x, q, step, bias, act=act)
    ref.assert_within(got, want)
    assert torch.equal(scnn.linear_int8_fwd(xq, q, step, bias, x_scale=xs, act=act), got)
