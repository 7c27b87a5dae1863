"""Global gradient norm and clipping on the GPU against their formulas in 64 bits."""
import math

import pytest
import torch

import paper_1801_10585_amd as scnn
from . import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LISTS = {"one": [1], "small": [3, 1, 7, 255], "empty_among": [0, 5, 0, 4097, 0], "chunks": [4096, 4097, 8191, 100000, 1],
         "layers": [(27, 1, 8), (8,), (27, 8, 16), (16,), (27, 16, 24), (24,)], "many": [17 + i for i in range(300)],
         "large": [3000001, 12, 2500000]}


def make(seed, shapes, dtypes, scale=0.1):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(s, generator=g) * scale).to(dtypes[i % len(dtypes)]).to(DEV) for i, s in enumerate(shapes)]


def expected(grads, max_norm):
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    return norm, min(1.0, max_norm / (norm + 1e-6))


def check(grads, outs, result, max_norm, before=None):
    before = before or grads
    norm, scale = expected(before, max_norm)
    got = result.cpu()
    # sums in fp64: n roundings of 2^-53 at most, n below 10^7
    assert float(got[0]) == pytest.approx(norm, rel=1e-9, abs=0) and float(got[1]) == pytest.approx(scale, rel=1e-9)
    for g, o in zip(before, outs):
        w = g.double() * scale
        # the scale rounded to fp32 and the product, then the type's own rounding
        ref.assert_within(o, (w.cpu(), ((2 * ref.U32 + ref.half(o.dtype)) * (1 + 1e-6) * w.abs() + ref.tiny(o.dtype)).cpu()))


@pytest.mark.parametrize("types", [(torch.float32,), (torch.bfloat16,), (torch.float16,), ref.TYPES], ids=str)
@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("max_norm", [0.05, 1e6, 0.0])
def test_clips_in_place_and_apart(name, types, max_norm):
    grads = make(len(name), LISTS[name], types)
    kept = [g.clone() for g in grads]
    outs = [torch.empty_like(g) for g in grads]
    result = scnn.clip_grad_norm(grads, max_norm, outs=outs)
    check(grads, outs, result, max_norm)
    assert all(torch.equal(a, b) for a, b in zip(grads, kept))
    again = scnn.clip_grad_norm(grads, max_norm)
    assert torch.equal(again, result) and all(torch.equal(a, b) for a, b in zip(grads, outs))
    assert float(scnn.grad_norm(kept)) == float(result[0])


def test_norm_of_large_and_small_entries():
    for v, n in ((1e30, 5000), (1e-30, 5000), (3e38, 9)):
        g = torch.full((n,), v, device=DEV)
        assert float(scnn.grad_norm([g])) == pytest.approx(float(g[0]) * math.sqrt(n), rel=1e-9)
    big = torch.full((70000,), 1e30, device=DEV)
    result = scnn.clip_grad_norm([big], 1.0)
    # (2^-24 for the scale, 2^-24 for the product)
    assert torch.allclose(big.cpu(), torch.full((70000,), 70000 ** -0.5), rtol=3e-7, atol=0) and float(result[1]) < 1e-30


def test_nan_and_infinity_show():
    a, b = torch.ones(10, device=DEV), torch.ones(5000, device=DEV)
    b[4999] = float("inf")
    result = scnn.clip_grad_norm([a, b], 1.0).cpu()
    assert math.isinf(float(result[0])) and float(result[1]) == 0.0
    assert not a.any() and bool(torch.isnan(b[4999])) and not b[:4999].any()
    a, b = torch.ones(10, device=DEV), torch.ones(5000, device=DEV)
    b[3] = float("nan")
    result = scnn.clip_grad_norm([a, b], 1.0).cpu()
    assert bool(torch.isnan(result).all()) and bool(torch.isnan(a).all()) and bool(torch.isnan(b).all())
    assert math.isnan(float(scnn.grad_norm([a])))


def test_views_and_orders_of_axes():
    base = torch.randn(3 * 40 * 50 + 7, device=DEV)
    flat = base.clone()
    grads = [base[1:2001].view(40, 50).t(), base[2003:4003].view(50, 40), base[4005:4006], base[4007:6007].view(2, 1000)]
    kept = [g.clone(memory_format=torch.preserve_format) for g in grads]
    result = scnn.clip_grad_norm(grads, 2.0)
    check(grads, grads, result, 2.0, before=kept)
    inside = torch.zeros_like(flat, dtype=torch.bool)
    for lo, hi in ((1, 2001), (2003, 4003), (4005, 4006), (4007, 6007)):
        inside[lo:hi] = True
    assert torch.equal(base[~inside], flat[~inside])  # what lies between the tensors stays


def test_refusals():
    g = torch.ones(100, device=DEV)
    for bad in ([g, g], [g[:50], g[40:]], [g, g[99:]]):
        with pytest.raises(scnn.ScnnError):
            scnn.clip_grad_norm(bad, 1.0)
    assert float(scnn.grad_norm([g, g])) == pytest.approx(200 ** 0.5)  # (only read: counts twice)
    with pytest.raises(scnn.ScnnError):
        scnn.clip_grad_norm([g[:50], g[50:]], 1.0, outs=[g[50:], g[:50]])
    for value in (-1.0, float("nan")):
        with pytest.raises(scnn.ScnnError):
            scnn.clip_grad_norm([g], value)
    with pytest.raises(ValueError):
        scnn.clip_grad_norm([g[::2]], 1.0)
    with pytest.raises(ValueError):
        scnn.clip_grad_norm([g], 1.0, outs=[torch.ones(99, device=DEV)])
    with pytest.raises(ValueError):
        scnn.clip_grad_norm([], 1.0)
    with pytest.raises(ValueError):
        scnn.clip_grad_norm([g.double()], 1.0)
    assert bool((g == 1).all())


def test_captured_and_replayed_and_another_stream():
    shapes = [(27, 8, 8), (8,), (130000,)]
    grads = make(1, shapes, (torch.float32,))
    outs = [torch.empty_like(g) for g in grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    result = scnn.clip_grad_norm(grads, 0.5, outs=outs, stream=side)
    torch.cuda.synchronize()
    check(grads, outs, result, 0.5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        result = scnn.clip_grad_norm(grads, 0.5, outs=outs)
    for k in range(4):
        for g, f in zip(grads, make(10 + k, shapes, (torch.float32,), scale=0.1 / 10 ** k)):
            g.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        check(grads, outs, result, 0.5)
