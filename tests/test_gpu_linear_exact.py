"""Products of linear layers whose results are known to the last bit: fp32 operands that need all three of their bf16 parts, and
whole numbers through the largest tiles."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# (rows, c_in, c_out).  Forward: few rows, w in registers, tiles of 64 x 64, those by four groups of waves, with k split too,
# 128 x 128; dx and dw: one pass of 32 and of 64 channels, then the same tiles
SIZES = [(3, 70, 40), (200, 24, 32), (500, 60, 50), (300, 100, 72), (70, 300, 130), (300, 270, 266), (65, 4100, 36), (3000, 70, 70),
         (2570, 520, 2560), (520, 2560, 2570), (2560, 2570, 520)]


def full(seed, *shape):
    """Odd 24-bit significands, signs, a few powers of two."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    m = torch.randint(1 << 22, 1 << 23, shape, generator=g, device=DEV) * 2 + 1
    e = torch.randint(-3, 4, shape, generator=g, device=DEV)
    s = torch.randint(0, 2, shape, generator=g, device=DEV) * 2 - 1
    return torch.ldexp((m * s).float(), e - 23)


def picks(seed, rows, cols, values=None):
    """One non-zero in every column: a power of two, or values[row, column]; and the row that holds it."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    at = torch.randint(0, rows, (cols,), generator=g, device=DEV)
    t = torch.zeros(rows, cols, device=DEV)
    n = torch.arange(cols, device=DEV)
    t[at, n] = torch.ldexp(torch.ones(cols, device=DEV), torch.randint(-2, 3, (cols,), generator=g, device=DEV)) if values is None else values[at, n]
    return t, at


def near(got, want):
    # products of two odd 24-bit numbers: what the six products of parts leave out is up to 2^-24 of values in 1 .. 4, their sums
    # are rounded at most five times, two of these by the whole
    assert float(((got.double() - want).abs() - 6 * ref.U32 * want.abs()).max()) <= 0


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_keeps_every_bit(size):
    rows, c_in, c_out = size
    x, w = full(1, rows, c_in), full(2, c_in, c_out)
    one, at = picks(3, c_in, c_out)
    assert torch.equal(scnn.linear_fwd(x, one), x[:, at] * one.sum(0))
    one, at = picks(4, c_in, rows)
    assert torch.equal(scnn.linear_fwd(one.t().contiguous(), w), w[at] * one.sum(0)[:, None])
    both, at = picks(5, c_in, c_out, values=w)
    near(scnn.linear_fwd(x, both), x[:, at].double() * both.double().sum(0))


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gradients_keep_every_bit(size):
    rows, c_in, c_out = size
    x, w = full(1, rows, c_in), full(2, c_in, c_out)
    # one product an element of dx: g has one channel a row
    one, at = picks(6, c_out, rows)
    dx, _, dbias = scnn.linear_bwd(x, w, one.t().contiguous())
    assert torch.equal(dx, w.t()[at] * one.sum(0)[:, None])
    assert torch.equal(dbias.double(), one.double().sum(1))  # (sums of powers of two: exact)
    one, at = picks(7, c_out, c_in)
    g = full(8, rows, c_out)
    dx, _, _ = scnn.linear_bwd(x, one.t().contiguous(), g)
    assert torch.equal(dx, g[:, at] * one.sum(0))
    # one product an element of dw: one row a channel
    one, at = picks(9, rows, c_out)
    _, dw, _ = scnn.linear_bwd(x, w, one)
    assert torch.equal(dw, x[at].t() * one.sum(0))
    one, at = picks(10, rows, c_in)
    _, dw, _ = scnn.linear_bwd(one, w, g)
    assert torch.equal(dw, g[at] * one.sum(0)[:, None])
    both, at = picks(11, rows, c_out, values=g)
    _, dw, _ = scnn.linear_bwd(x, w, both)
    near(dw, x[at].t().double() * both.double().sum(0))


def whole(seed, *shape, dtype):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=g, device=DEV).to(dtype)


def largest_tiles(m, n):
    """Whether 256 x 256 tiles are taken: two rounds of them or more, the rounds at least 95 per cent full."""
    tiles, units = -(-m // 256) * -(-n // 256), torch.cuda.get_device_properties(0).multi_processor_count
    rounds = -(-tiles // units)
    return rounds >= 2 and 20 * tiles >= 19 * rounds * units


HALVES = (torch.bfloat16, torch.float16)


@pytest.mark.parametrize("dtype", HALVES, ids=str)
@pytest.mark.parametrize("size", [(8100, 520, 4008), (8100, 1000, 6000), (4300, 576, 7640), (16300, 512, 2040)], ids=str)
def test_forward_by_tiles_of_256(size, dtype):
    """Edges on both sides, k that ends inside a step, a count on the device; sums below 2^24: exact before the one rounding."""
    rows, c_in, c_out = size
    assert largest_tiles(rows, c_out)
    x, w = whole(1, rows, c_in, dtype=dtype), whole(2, c_in, c_out, dtype=dtype)
    bias, residual = whole(3, c_out, dtype=dtype), whole(4, rows, c_out, dtype=dtype)
    z = x.double() @ w.double() + bias.double()
    out, pre = scnn.linear_fwd(x, w, bias, act="relu", residual=residual, keep_pre=True)
    want = (z.clamp(min=0) + residual.double()).to(dtype)
    assert torch.equal(pre, z.to(dtype)) and torch.equal(out, want)
    count = rows - 300
    x[count:] = float("nan")
    out, pre = torch.full_like(out, 5.0), torch.full_like(out, 5.0)
    scnn.linear_fwd(x, w, bias, act="relu", residual=residual, out=out, pre=pre, rows_dev=torch.tensor([count], device=DEV))
    assert torch.equal(out[:count], want[:count]) and torch.equal(pre[:count], z[:count].to(dtype))
    assert (out[count:] == 5).all() and (pre[count:] == 5).all()


@pytest.mark.parametrize("dtype", HALVES, ids=str)
def test_epilogue_of_tiles_of_256(dtype):
    rows, c_in, c_out = 8100, 520, 4008
    assert largest_tiles(rows, c_out)
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(rows, c_in, generator=g, device=DEV).to(dtype)
    w = (torch.randn(c_in, c_out, generator=g, device=DEV) * 0.06).to(dtype)
    bias, residual = torch.randn(c_out, generator=g, device=DEV).to(dtype), torch.randn(rows, c_out, generator=g, device=DEV).to(dtype)
    some = torch.cat([torch.arange(0, 40), torch.arange(4085, 4125), torch.arange(8060, 8100)]).to(DEV)
    for name in ("gelu", "silu"):
        out, pre = scnn.linear_fwd(x, w, bias, act=name, residual=residual, keep_pre=True)
        want, want_pre = ref.linear_fwd(x[some], w, bias, name, residual[some], dtype)
        ref.assert_within(out[some], want, "out")
        ref.assert_within(pre[some], want_pre, "pre")


@pytest.mark.parametrize("dtype", HALVES, ids=str)
def test_gradients_by_tiles_of_256(dtype):
    # dx: 8100 x 4008 over 520 channels; dw: 8100 x 4008 over 520 rows and fewer
    rows, c_in, c_out = 8100, 4008, 520
    assert largest_tiles(rows, c_in)
    x, w, g = whole(1, rows, c_in, dtype=dtype), whole(2, c_in, c_out, dtype=dtype), whole(3, rows, c_out, dtype=dtype)
    want = (g.double() @ w.double().t().contiguous()).to(dtype)
    dx, dw, _ = scnn.linear_bwd(x, w, g)
    assert torch.equal(dx, want)
    assert torch.equal(dw, (x.double().t().contiguous() @ g.double()).to(dtype))
    count = torch.tensor([8000], device=DEV)
    dx = torch.full_like(dx, 5.0)
    scnn.linear_bwd(x, w, g, want=(True, False, False), rows_dev=count, out=(dx, None, None))
    assert torch.equal(dx[:8000], want[:8000]) and (dx[8000:] == 5).all()
    rows, c_in, c_out = 520, 8100, 4008
    assert largest_tiles(c_in, c_out)
    x, w, g = whole(4, rows, c_in, dtype=dtype), whole(5, c_in, c_out, dtype=dtype), whole(6, rows, c_out, dtype=dtype)
    for count in (520, 512, 450, 3, 0):
        if count < 520:
            x[count:] = float("nan")
            g[count:] = float("inf")
        _, dw, dbias = scnn.linear_bwd(x, w, g, want=(False, True, True), rows_dev=torch.tensor([count], device=DEV))
        assert torch.equal(dw, (x[:count].double().t().contiguous() @ g[:count].double()).to(dtype)), count
        assert torch.equal(dbias, g[:count].double().sum(0).to(dtype)), count
