"""Calls of group norm, dropout and the 8-bit layers that users make besides the plain ones: several at once on streams of their own,
workspaces and results of the caller's, and what the binding refuses on GPU tensors."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import block_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def normal(seed, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def test_calls_on_two_streams_at_once():
    x, g, gamma = normal(1, 30000, 24), normal(2, 30000, 24), normal(3, 24)
    xs, w = normal(4, 300, 2000, dtype=torch.bfloat16), scnn.quantize_weight(normal(5, 2000, 500, dtype=torch.bfloat16))
    offsets = torch.tensor([0, 11111, 30000], device=DEV)

    def calls(k, stream=None):
        y, m, r = scnn.group_norm_fwd(x, 4, gamma, offsets=offsets, act="gelu", stream=stream)
        back = scnn.group_norm_bwd(x, g, 4, gamma, None, m, r, offsets=offsets, act="gelu", stream=stream)
        d = scnn.dropout_fwd(x, 0.3, seed=k, residual=g, stream=stream)
        return [y, m, r, *back, d, scnn.linear_int8_fwd(xs, *w, act="silu", stream=stream)]

    want = [calls(k) for k in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = [calls(k, streams[k]) for k in range(2)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_workspaces_of_the_callers_and_too_small_ones():
    x = normal(6, 20000, 24, dtype=torch.float16)
    need = scnn.group_norm_fwd_workspace(torch.float16, 20000, 1, 24, 4)
    assert need > 256
    want = scnn.group_norm_fwd(x, 4)
    # (larger than asked for, full of something)
    ws = torch.full((need + 512,), 255, dtype=torch.uint8, device=DEV)
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(scnn.group_norm_fwd(x, 4, workspace=ws), want))
    with pytest.raises(scnn.ScnnError, match="workspace"):
        scnn.group_norm_fwd(x, 4, workspace=ws[:need - 256])
    need = scnn.group_norm_bwd_workspace(torch.float16, 20000, 1, 24, 4)
    back = scnn.group_norm_bwd(x, x, 4, None, None, *want[1:])
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)
    assert all(torch.equal(a, b) for a, b in zip(scnn.group_norm_bwd(x, x, 4, None, None, *want[1:], workspace=ws), back))
    q = scnn.quantize_weight(normal(7, 4096, 40, dtype=torch.float16))
    rows = normal(8, 50, 4096, dtype=torch.float16)
    need = scnn.linear_int8_fwd_workspace(torch.float16, 50, 4096, 40)
    assert need > scnn.linear_int8_fwd_workspace(torch.float16, 50, 4096, 40, given=True) > 256  # (a split sum)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)
    assert torch.equal(scnn.linear_int8_fwd(rows, *q, workspace=ws), scnn.linear_int8_fwd(rows, *q))
    with pytest.raises(scnn.ScnnError, match="workspace"):
        scnn.linear_int8_fwd(rows, *q, workspace=ws[:need - 256])


def test_samples_alone_and_together_agree():
    """A sample's results do not hang on its place in the batch but for the last bits of other blocks of rows."""
    x, gamma = normal(9, 5000, 16), normal(10, 16)
    cuts = [0, 1, 700, 700, 4999, 5000]
    out, mean, rstd = scnn.group_norm_fwd(x, 4, gamma, offsets=torch.tensor(cuts, device=DEV), act="silu")
    for b, (lo, hi) in enumerate(zip(cuts, cuts[1:])):
        if hi > lo:
            y, m, r = scnn.group_norm_fwd(x[lo:hi], 4, gamma, act="silu")
            # both are roundings of sums in fp64: one step of fp32 apart at most, and what a step of rstd or mean makes of it
            assert torch.allclose(m[0], mean[b], rtol=2 * ref.U32, atol=1e-30) and torch.allclose(r[0], rstd[b], rtol=4 * ref.U32, atol=0)
            assert torch.allclose(y, out[lo:hi], rtol=16 * ref.U32, atol=16 * ref.U32 * float(x.abs().max() * r.max()))


def test_large_products_captured_first_and_replayed():
    """The largest tiles need more on-chip memory than a kernel has by itself: their first call may be a captured one."""
    m = 8192
    x, w = normal(11, m, 2048, dtype=torch.bfloat16), scnn.quantize_weight(normal(12, 2048, 2048, dtype=torch.bfloat16))
    out = torch.empty(m, 2048, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(scnn.linear_int8_fwd_workspace(torch.bfloat16, m, 2048, 2048), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        scnn.linear_int8_fwd(x, *w, out=out, workspace=ws)
    for k in range(3):
        x.copy_(normal(20 + k, m, 2048, dtype=torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, scnn.linear_int8_fwd(x, *w))
        xq, xs = scnn.quantize_rows(x[-300:])
        ref.assert_within(out[-300:], ref.linear_int8(xq, xs, *w, None, "none", None, torch.bfloat16))


def test_refusals_of_the_binding():
    x, i64 = normal(13, 12, 8), torch.int64
    good = torch.tensor([0, 5, 12], device=DEV)
    out, mean, rstd = scnn.group_norm_fwd(x, 2, offsets=good)
    bad = [lambda: scnn.group_norm_fwd(x, 2, offsets=good.to(torch.int32)), lambda: scnn.group_norm_fwd(x, 2, offsets=good.cpu()),
           lambda: scnn.group_norm_fwd(x, 2, offsets=good[:1]), lambda: scnn.group_norm_fwd(x, 2, offsets=good, batch=3),
           lambda: scnn.group_norm_fwd(x, 2, gamma=x[0, :7]), lambda: scnn.group_norm_fwd(x, 2, beta=x[0].half()),
           lambda: scnn.group_norm_fwd(x, 2, act="tanh"), lambda: scnn.group_norm_fwd(x.to(torch.float64), 2),
           lambda: scnn.group_norm_fwd(x, 2, out=(x.t().contiguous().t(), mean[:1], rstd[:1])),
           lambda: scnn.group_norm_bwd(x, x, 2, None, None, mean[0], rstd[0]),
           lambda: scnn.group_norm_bwd(x, x, 2, None, None, mean, rstd[:1], offsets=good),
           lambda: scnn.group_norm_bwd(x, x[:5], 2, None, None, mean, rstd, offsets=good),
           lambda: scnn.sample_offsets(x, 2), lambda: scnn.sample_offsets(x.to(torch.int32), 0), lambda: scnn.sample_offsets(x.to(torch.int32), 1 << 40),
           lambda: scnn.dropout_fwd(x, 0.5, seed=-1), lambda: scnn.dropout_fwd(x, 0.5, offset=1 << 64),
           lambda: scnn.dropout_fwd(x, 0.5, rng=good), lambda: scnn.dropout_fwd(x, 0.5, rng=good[:2].float()),
           lambda: scnn.dropout_fwd(x, 0.5, residual=x[:3]), lambda: scnn.dropout_bwd(x[0], 0.5),
           lambda: scnn.quantize_rows(x[0]), lambda: scnn.quantize_weight(x.to(i64))]
    q, s = scnn.quantize_weight(x)
    xq, xs = scnn.quantize_rows(normal(14, 3, 12))
    bad += [lambda: scnn.linear_int8_fwd(xq, q, s), lambda: scnn.linear_int8_fwd(xq, q, s, x_scale=xs),  # no scale; no type
            lambda: scnn.linear_int8_fwd(normal(14, 3, 100), q, s), lambda: scnn.linear_int8_fwd(normal(14, 3, 12), q[:, :12], s),
            lambda: scnn.linear_int8_fwd(normal(14, 3, 12), q, s[:7]), lambda: scnn.linear_int8_fwd(normal(14, 3, 12), q.float(), s),
            lambda: scnn.linear_int8_fwd(normal(14, 3, 12).to(torch.float64), q, s), lambda: scnn.linear_int8_fwd(normal(14, 3, 12), q, s, dtype=torch.float16),
            lambda: scnn.linear_int8_fwd(xq[:, :32].contiguous(), q, s, x_scale=xs, dtype=torch.float32),
            lambda: scnn.linear_int8_fwd(normal(14, 3, 12), q[0], s), lambda: scnn.linear_int8_fwd(normal(14, 3, 12), q, s, bias=s.half())]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")
    for call in (lambda: scnn.group_norm_fwd(x, 3), lambda: scnn.group_norm_fwd(x, 2, batch=5), lambda: scnn.group_norm_fwd(x, 2, eps=-1.0),
                 lambda: scnn.group_norm_fwd(x, 0), lambda: scnn.group_norm_fwd(x, 2, batch=0), lambda: scnn.group_norm_fwd(x, 2, batch=-1), lambda: scnn.group_norm_fwd(x, -2), lambda: scnn.dropout_fwd(x, 1.5),
                 lambda: scnn.dropout_fwd(x, float("nan")), lambda: scnn.group_norm_fwd(x, 2, out=(x, mean[:1], rstd[:1]))):
        with pytest.raises(scnn.ScnnError):
            call()


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=str)
def test_calls_of_many_samples(dtype):
    """Calls of more than 2^24 values, of equal samples with and without offsets, of short ones whole and in two halves."""
    e = torch.finfo(dtype).eps
    x, g, gamma = normal(15, 300000, 64, dtype=dtype), normal(16, 300000, 64, dtype=dtype), normal(17, 64, dtype=dtype)

    def both(x, g, batch=None, offsets=None):
        y, m, r = scnn.group_norm_fwd(x, 8, gamma, batch=batch, offsets=offsets, act="silu")
        return [y, m, r, *scnn.group_norm_bwd(x, g, 8, gamma, None, m, r, offsets=offsets, act="silu")]

    same = both(x, g, batch=600), both(x, g, offsets=torch.arange(0, 300001, 500, device=DEV))
    for k, (a, b) in enumerate(zip(*same)):
        # sums in other orders: steps of fp32 apart before the rounding (64 of them where a term cancels or 300000 are added), then one step of the type
        near = (64 if k < 4 else 4096) * ref.U32 * float(b.float().abs().max())
        assert torch.allclose(a.float(), b.float(), rtol=e if k != 1 and k != 2 else 8 * ref.U32, atol=near), k
    cuts = torch.sort(torch.randint(0, 150001, (1, 3000), generator=torch.Generator().manual_seed(1)), 1)[0][0].to(DEV)
    half = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), cuts, torch.full((1,), 150000, device=DEV)])
    whole = both(x, g, offsets=torch.cat([half, half[1:] + 150000]))
    for k, one in enumerate((both(x[:150000], g[:150000], offsets=half), both(x[150000:], g[150000:], offsets=half))):
        at = slice(k * 150000, (k + 1) * 150000), slice(k * 3001, (k + 1) * 3001)
        for a, b, rows in ((whole[0], one[0], 0), (whole[3], one[3], 0), (whole[1], one[1], 1), (whole[2], one[2], 1)):
            assert torch.equal(a[at[rows]], b)
