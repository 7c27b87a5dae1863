"""Every kernel that an 8-bit layer may be given to, at sizes that cut its tiles and steps: one row with one, two and four columns a
wave; tiles of 128 with whole and split k; tiles of 256.  (The rule is int8_plan's, on 256 compute units.)"""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import block_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = (torch.float32, torch.bfloat16, torch.float16)
# a row's two and four columns a wave begin at 2048 and 4096; 20000: parts of 16384
ROW = [(1, 300, 2047), (1, 1001, 2051), (1, 4096, 4101), (1, 20000, 5003)]
# rows of 17 half steps of 128 bytes, of 193 in four splits; last tiles of 56 rows and 84 columns, of 104 and 105
RING128 = [(3000, 1030, 2900), (1000, 12290, 1001)]
# rows of 33 half steps, last tiles of 164 rows and 251 columns; of 20 whole steps, 225 and 248
RING256 = [(8100, 2100, 2043), (7905, 2500, 2040)]


def moved(t):
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("size", ROW + RING128 + RING256, ids=str)
def test_matches_the_formula(size, dtype):
    rows, c_in, c_out = size
    gen = torch.Generator().manual_seed(rows + c_out)

    def normal(*shape, s=1.0):
        return (torch.randn(*shape, generator=gen) * s).to(dtype).to(DEV)

    x, bias, residual = normal(rows, c_in), normal(c_out, s=0.3), normal(rows, c_out)
    q, steps = scnn.quantize_weight(normal(c_in, c_out, s=c_in ** -0.5))
    xq, xs = scnn.quantize_rows(x)
    want_q, want_s = ref.quantize(x)
    assert torch.equal(xq[:, :c_in].cpu(), want_q) and not xq[:, c_in:].any() and torch.equal(xs.cpu(), want_s)
    out = None
    for b, act, r in ((None, "none", None), (bias, "relu", None), (None, "silu", residual), (bias, "gelu", residual)):
        want = ref.linear_int8(xq, xs, q, steps, b, act, r, dtype)
        out = scnn.linear_int8_fwd(x, q, steps, b, act=act, residual=r)
        ref.assert_within(out, want, act)
        given = scnn.linear_int8_fwd(xq, q, steps, b, x_scale=xs, act=act, residual=r, dtype=dtype)
        assert torch.equal(given, out), act
    # bias, results and the residual that they replace at any element
    place = moved(residual)
    assert scnn.linear_int8_fwd(moved(x), q, moved(steps), moved(bias), act="gelu", residual=place, out=place) is place
    assert torch.equal(place, out)
    # a row count on the device that ends inside a tile, no row, and more than there are
    for count in (rows - rows // 3, 1, 0, 1 << 40):
        n = min(count, rows)
        some = torch.full((rows, c_out), 7.0, dtype=dtype, device=DEV)
        bad = x.clone()
        bad[n:] = float("nan")
        scnn.linear_int8_fwd(bad, q, steps, bias, act="gelu", residual=residual, rows_dev=torch.tensor([count], device=DEV), out=some)
        assert torch.equal(some[:n], out[:n]) and bool((some[n:] == 7).all()), count


@pytest.mark.parametrize("size", ROW[2:] + RING128 + RING256, ids=str)
def test_sums_are_exact(size):
    """Largest magnitudes of either sign, in sums that end near 2^31 where k is long."""
    rows, c_in, c_out = size
    gen = torch.Generator().manual_seed(c_in)
    width = scnn.int8_row_bytes(c_in)
    x, w = torch.zeros(rows, width, dtype=torch.int8), torch.zeros(c_out, width, dtype=torch.int8)
    x[:, :c_in] = torch.randint(-128, 128, (rows, c_in), generator=gen)
    w[:, :c_in] = torch.randint(-128, 128, (c_out, c_in), generator=gen)
    x[-1, :c_in], w[0, :c_in], w[-1, :c_in] = -128, -128, 127
    total = (x.double().to(DEV) @ w.double().to(DEV).t().contiguous()).cpu()  # (whole numbers below 2^53: exact in any order)
    one = torch.ones(max(rows, c_out), device=DEV)
    got = scnn.linear_int8_fwd(x.to(DEV), w.to(DEV), one[:c_out], x_scale=one[:rows], dtype=torch.float32)
    assert torch.equal(got.cpu(), total.float())


@pytest.mark.parametrize("size", RING128 + RING256[:1], ids=str)
def test_captured_and_replayed(size):
    rows, c_in, c_out = size
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(rows, c_in, generator=gen).to(torch.bfloat16).to(DEV)
    q = scnn.quantize_weight(torch.randn(c_in, c_out, generator=gen).to(torch.bfloat16).to(DEV))
    out = torch.empty(rows, c_out, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(scnn.linear_int8_fwd_workspace(torch.bfloat16, *size), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        scnn.linear_int8_fwd(x, *q, act="silu", out=out, workspace=ws)
    for k in range(3):
        x.copy_(torch.randn(rows, c_in, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, scnn.linear_int8_fwd(x, *q, act="silu"))
