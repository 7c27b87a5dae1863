"""Dropout on the GPU: the mask against the published generator, values, gradients, replays."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import block_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def normal(seed, rows, channels, dtype):
    return torch.randn(rows, channels, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def kept(rows, channels, p, seed, offset):
    return (ref.words(0, rows * channels, seed, offset) >= round(p * 65536)).view(rows, channels)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,channels", [(1, 1), (3, 2), (1, 7), (5, 8), (17, 9), (100, 25), (33, 64), (7, 1001)])
def test_values_mask_and_gradient(rows, channels, dtype):
    x, r = normal(1, rows, channels, dtype), normal(2, rows, channels, dtype)
    for p, seed, offset in ((0.5, 0, 0), (0.1, 12345, 7), (0.37, (1 << 64) - 1, (1 << 64) - 2), (0.9, 1 << 32, 1 << 63)):
        k = kept(rows, channels, p, seed, offset)
        got = scnn.dropout_fwd(x, p, seed=seed, offset=offset)
        ref.assert_within(got, ref.dropout(x, p, k, None, dtype))
        assert torch.equal(got.cpu() != 0, k & (x.cpu() != 0))
        ref.assert_within(scnn.dropout_fwd(x, p, seed=seed, offset=offset, residual=r), ref.dropout(x, p, k, r, dtype))
        assert torch.equal(scnn.dropout_bwd(x, p, seed=seed, offset=offset), got)


def test_words_to_the_last_bit():
    n, seed, offset = 200, 0x0123456789abcdef, 0xfedcba9876543210
    want = ref.words(0, n, seed, offset)
    x = torch.ones(1, n, device=DEV)
    low, high = torch.zeros(n, dtype=torch.int64), torch.full((n,), 65536)
    for _ in range(16):  # the largest threshold that keeps a value, by halving: a value's threshold at each turn
        mid = (low + high) // 2
        keep = torch.zeros(n, dtype=torch.bool)
        for t in mid.unique().tolist():
            got = scnn.dropout_fwd(x, t / 65536, seed=seed, offset=offset).cpu()[0] != 0
            keep = torch.where(mid == t, got, keep)
        low, high = torch.where(keep, mid, low), torch.where(keep, high, mid)
    assert torch.equal(low, want)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_nothing_and_everything_dropped(dtype):
    x, r = normal(3, 50, 33, dtype), normal(4, 50, 33, dtype)
    assert torch.equal(scnn.dropout_fwd(x, 0.0, seed=5), x)
    assert torch.equal(scnn.dropout_fwd(x, 2.0 ** -18, seed=5), x)  # (less than half a step)
    assert not scnn.dropout_fwd(x, 1.0, seed=5).any()
    assert torch.equal(scnn.dropout_fwd(x, 1.0, seed=5, residual=r), r)
    # what is dropped is dropped, whatever it was
    bad = torch.full_like(x, float("nan"))
    bad[:, ::2] = float("inf")
    k = kept(50, 33, 0.5, 5, 0)
    got = scnn.dropout_fwd(bad, 0.5, seed=5).cpu()
    assert not got[~k].any() and bool((torch.isnan(got[k]) | torch.isinf(got[k])).all())


def test_share_of_values_kept_and_independence():
    x = torch.ones(1000, 1000, device=DEV)
    a, b, c = (scnn.dropout_fwd(x, 0.3, seed=seed, offset=offset).cpu() != 0 for seed, offset in ((1, 1), (1, 2), (2, 1)))
    # a million draws: five standard deviations are 0.0023
    for m in (a, b, c):
        assert abs(float(m.float().mean()) - 0.7) < 0.0023 + 2 ** -17
    for m in (a & b, a & c, b & c):
        assert abs(float(m.float().mean()) - 0.49) < 0.0025 + 2 ** -16


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("count", [37, 0, -3, 1 << 40])
def test_row_count_from_the_device(count, dtype):
    cap, channels = 90, 25
    n = max(0, min(cap, count))
    x = normal(6, cap, channels, dtype)
    want = scnn.dropout_fwd(x, 0.4, seed=9)
    x[n:] = float("nan")
    out = torch.full((cap, channels), 7.0, dtype=dtype, device=DEV)
    rows_dev = torch.tensor([count], device=DEV)
    scnn.dropout_fwd(x, 0.4, seed=9, rows_dev=rows_dev, out=out)
    assert torch.equal(out[:n], want[:n]) and bool((out[n:] == 7).all())
    out.fill_(7)
    scnn.dropout_bwd(x, 0.4, seed=9, rows_dev=rows_dev, out=out)
    assert torch.equal(out[:n], want[:n]) and bool((out[n:] == 7).all())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_in_place_any_start_and_strides(dtype):
    rows, channels = 301, 35
    x, r = normal(7, rows, channels, dtype), normal(8, rows, channels, dtype)
    want, with_r = scnn.dropout_fwd(x, 0.25, seed=3, offset=4), scnn.dropout_fwd(x, 0.25, seed=3, offset=4, residual=r)
    flat = torch.empty(rows * channels + 1, dtype=dtype, device=DEV)
    flat[1:] = x.view(-1)
    v = flat[1:].view(rows, channels)
    assert torch.equal(scnn.dropout_fwd(v, 0.25, seed=3, offset=4), want)
    assert torch.equal(scnn.dropout_fwd(x.t().contiguous().t(), 0.25, seed=3, offset=4), want)
    assert scnn.dropout_fwd(v, 0.25, seed=3, offset=4, out=v) is v and torch.equal(v, want)
    q = r.clone()
    scnn.dropout_fwd(x, 0.25, seed=3, offset=4, residual=q, out=q)
    assert torch.equal(q, with_r)
    q = x.clone()
    scnn.dropout_fwd(q, 0.25, seed=3, offset=4, residual=r, out=q)
    assert torch.equal(q, with_r)
    q = x.clone()
    scnn.dropout_bwd(q, 0.25, seed=3, offset=4, out=q)
    assert torch.equal(q, want)
    assert scnn.dropout_fwd(x[:0], 0.25).shape == (0, channels)


def test_values_past_32_bits():
    rows, channels = (1 << 20) + 3, 4096
    x = torch.ones(rows, channels, dtype=torch.bfloat16, device=DEV)
    scnn.dropout_fwd(x, 0.5, seed=77, offset=88, out=x)
    first = (rows - 2) * channels
    assert first > 1 << 32
    want = ref.words(first, 2 * channels, 77, 88) >= 32768
    assert torch.equal((x[-2:] != 0).view(-1).cpu(), want)
    some = x[-4096:].cpu() != 0  # (2^24 draws: five standard deviations are 0.0006)
    assert abs(float(some.float().mean(dtype=torch.float64)) - 0.5) < 0.0007


def test_captured_with_seed_and_offset_from_the_device_and_another_stream():
    x, r = normal(11, 200, 35, torch.float32), normal(12, 200, 35, torch.float32)
    rng = torch.tensor([5, 6], dtype=torch.int64, device=DEV)
    out, back = torch.empty_like(x), torch.empty_like(x)

    def step(stream=None):
        scnn.dropout_fwd(x, 0.3, rng=rng, residual=r, out=out, stream=stream)
        scnn.dropout_bwd(r, 0.3, rng=rng, out=back, stream=stream)

    def want(offset):
        return scnn.dropout_fwd(x, 0.3, seed=5, offset=offset, residual=r), scnn.dropout_bwd(r, 0.3, seed=5, offset=offset)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((out, back), want(6)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        rng[1:].add_(1)
    masks = []
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, back), want(6 + k)))
        masks.append(back != 0)
    assert not torch.equal(masks[0], masks[1])
    whole = torch.tensor([-1, 1 << 62], dtype=torch.int64, device=DEV)  # (as unsigned numbers)
    assert torch.equal(scnn.dropout_fwd(x, 0.3, rng=whole), scnn.dropout_fwd(x, 0.3, seed=(1 << 64) - 1, offset=1 << 62))
