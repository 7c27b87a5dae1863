"""Layers on rows of values at the largest extents that the calls take: launches of 2^32 threads and more along an axis."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def room(gib):
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip(f"needs {gib} GiB of device memory")


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("channels,dtype", [((1 << 25) + 5, torch.float32), (1 << 28, torch.bfloat16)], ids=str)
def test_gradients_of_one_long_norm(channels, dtype):
    room(24)
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(1, channels, generator=gen, device=DEV).to(dtype)
    g = torch.randn(1, channels, generator=gen, device=DEV).to(dtype)
    gamma = torch.rand(channels, generator=gen, device=DEV).to(dtype)
    y, mean, rstd = scnn.layer_norm_fwd(x, gamma, None)
    dx, dgamma, dbeta = scnn.layer_norm_bwd(x, g, gamma, mean, rstd)
    m, r = mean.double(), rstd.double()
    # rows' sums: 1024 threads, each over channels / 1024 values in turn
    n = (64 + channels / 1024) * ref.U32
    for lo in range(0, channels, 1 << 26):
        part = slice(lo, min(channels, lo + (1 << 26)))
        xh, gg, ga = (x[0, part].double() - m) * r, g[0, part].double(), gamma[part].double()
        for got, want, slack in ((dgamma[part], gg * xh, 8 * ref.U32), (dbeta[part], gg, 0.0), (y[0, part], xh * ga, 8 * ref.U32)):
            assert float(((got.double() - want).abs() - (ref.half(dtype) + slack) * want.abs()).max()) <= 4 * ref.U32 * float(m.abs() * r) + ref.tiny(dtype)
    h = g.double() * gamma.double()
    xh = (x.double() - m) * r
    m_h, m_hx, a_h, a_hx = h.mean(), (h * xh).mean(), h.abs().mean(), (h * xh).abs().mean()
    want = r * (h - m_h - xh * m_hx)
    bound = r * (8 * ref.U32 * (h.abs() + m_h.abs() + (xh * m_hx).abs()) + n * (a_h + xh.abs() * a_hx)) + ref.half(dtype) * want.abs() + ref.tiny(dtype)
    assert float(((dx.double() - want).abs() - bound).max()) <= 0


def test_bias_gradient_of_the_widest_layer():
    room(24)
    c_out = 1 << 28
    gen = torch.Generator(device=DEV).manual_seed(2)
    g = torch.randint(-8, 9, (2, c_out), generator=gen, device=DEV, dtype=torch.int8).to(torch.bfloat16)
    x = torch.tensor([[2.0], [-1.0]], device=DEV, dtype=torch.bfloat16)
    w = torch.zeros(1, c_out, device=DEV, dtype=torch.bfloat16)
    w[0, -5:] = torch.tensor([1.0, 2.0, -1.0, 4.0, 3.0])
    dx, dw, dbias = scnn.linear_bwd(x, w, g)
    assert torch.equal(dbias, g[0] + g[1]) and torch.equal(dw[0], 2 * g[0] - g[1])  # (whole numbers up to 24: exact)
    assert torch.equal(dx[:, 0].float(), (g[:, -5:].float() * w[0, -5:].float()).sum(1).bfloat16().float())
    # one row of fp32, k of a few and of one (whole numbers)
    w = torch.randint(-8, 9, (1, c_out), generator=gen, device=DEV, dtype=torch.int8).float()
    assert torch.equal(scnn.linear_fwd(torch.full((1, 1), 3.0, device=DEV), w), 3 * w)


@pytest.mark.parametrize("c_in", [1, 8], ids=["staged", "copied"])
def test_more_rows_than_a_launch_has_tiles_along_one_axis(c_in):
    room(130)
    rows, c_out = (1 << 30) + 70, 40
    x = torch.zeros(rows, c_in, device=DEV, dtype=torch.bfloat16)
    x[:, 0] = torch.arange(rows, device=DEV, dtype=torch.int32).remainder_(251).to(torch.bfloat16)  # (up to 250: exact)
    w = torch.zeros(c_in, c_out, device=DEV, dtype=torch.bfloat16)
    w[0] = torch.tensor([1.0, -1.0, 2.0, 0.0, 0.5] * 8)
    out = torch.empty(rows, c_out, device=DEV, dtype=torch.bfloat16)
    out[-64:] = 7.0
    scnn.linear_fwd(x, w, out=out)
    for lo in range(0, rows, 1 << 27):
        assert torch.equal(out[lo:lo + (1 << 27)], x[lo:lo + (1 << 27), :1] * w[:1]), lo


def test_a_split_sum_of_more_results_than_a_launch_joins_along_one_axis():
    room(90)
    rows, c_in, c_out = 1 << 16, 65600, 1 << 16  # (2^32 results, two parts of k)
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randint(-1, 2, (rows, c_in), generator=gen, device=DEV, dtype=torch.int8).to(torch.bfloat16)
    w = torch.randint(-1, 2, (c_in, c_out), generator=gen, device=DEV, dtype=torch.int8).to(torch.bfloat16)
    out = scnn.linear_fwd(x, w)
    assert scnn.linear_fwd_workspace(torch.bfloat16, rows, c_in, c_out) > 2 * 4 * rows * c_out
    some = torch.cat([torch.arange(0, 8), torch.arange(32764, 32772), torch.arange(rows - 8, rows)]).to(DEV)
    want = torch.zeros(len(some), c_out, device=DEV, dtype=torch.float64)
    for lo in range(0, c_in, 8200):  # (whole numbers: exact in any order)
        want += x[some, lo:lo + 8200].float() @ w[lo:lo + 8200].float()
    assert torch.equal(out[some], want.to(torch.bfloat16))
    del want
    want = torch.zeros(rows, 24, device=DEV, dtype=torch.float64)
    for lo in range(0, c_in, 8200):
        want += x[:, lo:lo + 8200].float() @ w[lo:lo + 8200][:, some].float()
    assert torch.equal(out[:, some], want.to(torch.bfloat16))
