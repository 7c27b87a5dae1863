"""Layer norm (forward and gradients) on the GPU against its formulas in 64 bits."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# (rows, channels): every width of the kernels' row groups with its neighbours, odd widths, rows past a workgroup's registers
SIZES = [(1, 1), (5, 2), (700, 3), (1, 1024), (3, 4), (65, 5), (1000, 8), (129, 9), (300, 17), (2000, 25), (777, 32), (50, 33),
         (400, 64), (33, 65), (64, 127), (20, 256), (9, 257), (31, 511), (12, 513), (40, 1025), (7, 2049), (5, 4096), (3, 4097),
         (3, 8193), (2, 16385), (300, 9001), (2, 33001), (1, 70000)]


def make(seed, rows, channels, dtype, shift=0.5):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, s=1.0, m=0.0):
        return (torch.randn(*shape, generator=g) * s + m).to(dtype).to(DEV)

    return {"x": normal(rows, channels, s=1.5, m=shift), "gamma": normal(channels, s=0.2, m=1.0), "beta": normal(channels, s=0.3),
            "g": normal(rows, channels, s=0.5)}


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("k,size", list(enumerate(SIZES)), ids=str)
def test_matches_the_formulas(k, size, dtype):
    d = make(k, *size, dtype)
    for gamma, beta in ((d["gamma"], d["beta"]), (None, None), (d["gamma"], None)):
        got = scnn.layer_norm_fwd(d["x"], gamma, beta, eps=1e-5)
        for what, a, b in zip(("out", "mean", "rstd"), got, ref.layer_norm_fwd(d["x"], gamma, beta, 1e-5, dtype)):
            ref.assert_within(a, b, what)
        back = scnn.layer_norm_bwd(d["x"], d["g"], gamma, got[1], got[2])
        want = ref.layer_norm_bwd(d["x"], d["g"], gamma, got[1], got[2], dtype)
        for what, a, b in zip(("dx", "dgamma", "dbeta"), back, want):
            ref.assert_within(a, b, what)
        for a, b in zip(scnn.layer_norm_bwd(d["x"], d["g"], gamma, got[1], got[2]), back):
            assert torch.equal(a, b)
    for i in range(3):
        one = scnn.layer_norm_bwd(d["x"], d["g"], d["gamma"], got[1], got[2], want=[i == j for j in range(3)])
        assert [o is None for o in one] == [i != j for j in range(3)] and torch.equal(one[i], back[i])


def test_gradients_match_differences():
    d = {k: v.cpu().double() for k, v in make(3, 4, 6, torch.float32).items()}

    def loss(x, gamma, beta):
        m = x.mean(1, keepdim=True)
        v = ((x - m) ** 2).mean(1, keepdim=True)
        return (((x - m) / torch.sqrt(v + 1e-5) * gamma + beta) * d["g"]).sum()

    f = {k: v.float().to(DEV) for k, v in d.items()}
    _, mean, rstd = scnn.layer_norm_fwd(f["x"], f["gamma"], f["beta"])
    got = scnn.layer_norm_bwd(f["x"], f["g"], f["gamma"], mean, rstd)
    h = 1e-5
    for i, key in enumerate(("x", "gamma", "beta")):
        args = [d["x"], d["gamma"], d["beta"]]
        for at in range(args[i].numel()):
            e = torch.zeros_like(args[i]).view(-1)
            e[at] = h
            hi = [a + e.view_as(a) if j == i else a for j, a in enumerate(args)]
            lo = [a - e.view_as(a) if j == i else a for j, a in enumerate(args)]
            slope = (loss(*hi) - loss(*lo)) / (2 * h)
            # 64-bit cancellation over h, h^2 times third derivatives below 100, and some tens of fp32 roundings of size 3
            assert abs(float(got[i].view(-1)[at]) - float(slope)) < 2e-5, (key, at)


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
def test_rows_of_equal_values_and_far_from_zero(dtype):
    x = torch.full((9, 40), 3.0, dtype=dtype, device=DEV)
    x[1] = 0
    x[2] = torch.finfo(dtype).max / 64
    out, mean, rstd = scnn.layer_norm_fwd(x, eps=1e-3)
    assert not out.any() and float(mean[0]) == 3.0 and float(mean[1]) == 0.0
    assert torch.allclose(rstd.cpu(), torch.full((9,), 1e-3 ** -0.5))
    if dtype == torch.float32:
        far = make(5, 6, 300, dtype, shift=1000.0)
        for a, b in zip(scnn.layer_norm_fwd(far["x"]), ref.layer_norm_fwd(far["x"], None, None, 1e-5, dtype)):
            ref.assert_within(a, b)


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("channels", [20, 600, 40000])
def test_nan_and_infinities_stay_in_their_rows(dtype, channels):
    d = make(7, 6, channels, dtype)
    clean = scnn.layer_norm_fwd(d["x"], d["gamma"], d["beta"])[0]
    d["x"][1, 3] = float("nan")
    d["x"][4, channels - 1] = float("inf")
    out, mean, rstd = scnn.layer_norm_fwd(d["x"], d["gamma"], d["beta"])
    for r in range(6):
        if r in (1, 4):
            assert bool(torch.isnan(out[r]).all())
        else:
            assert torch.equal(out[r], clean[r])
    dx = scnn.layer_norm_bwd(d["x"], d["g"], d["gamma"], mean, rstd)[0]
    assert [bool(torch.isnan(dx[r]).any()) for r in range(6)] == [False, True, False, False, True, False]


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("channels", [25, 64, 700, 5000, 20000])
@pytest.mark.parametrize("cap,count", [(90, 37), (90, 0), (90, -3), (90, 1 << 40)])
def test_row_count_from_the_device(cap, count, channels, dtype):
    n = max(0, min(cap, count))
    d = make(11, cap, channels, dtype)
    d["x"][n:] = float("nan")
    d["g"][n:] = float("nan")
    rows_dev = torch.tensor([count], dtype=torch.int64, device=DEV)
    out = torch.full((cap, channels), 7.0, dtype=dtype, device=DEV)
    mean, rstd = torch.full((cap,), 8.0, device=DEV), torch.full((cap,), 9.0, device=DEV)
    scnn.layer_norm_fwd(d["x"], d["gamma"], d["beta"], rows_dev=rows_dev, out=(out, mean, rstd))
    assert bool((out[n:] == 7).all()) and bool((mean[n:] == 8).all()) and bool((rstd[n:] == 9).all())
    if n:
        for a, b in zip((out, mean, rstd), ref.layer_norm_fwd(d["x"][:n], d["gamma"], d["beta"], 1e-5, dtype)):
            ref.assert_within(a[:n], b)
    dx = torch.full((cap, channels), 7.0, dtype=dtype, device=DEV)
    dgamma, dbeta = (torch.full((channels,), 5.0, dtype=dtype, device=DEV) for _ in range(2))
    scnn.layer_norm_bwd(d["x"], d["g"], d["gamma"], mean, rstd, rows_dev=rows_dev, out=(dx, dgamma, dbeta))
    assert bool((dx[n:] == 7).all())
    for a, b in zip((dx[:n], dgamma, dbeta), ref.layer_norm_bwd(d["x"][:n], d["g"][:n], d["gamma"], mean[:n], rstd[:n], dtype)):
        ref.assert_within(a, b)


def test_no_rows():
    x = torch.empty((0, 12), device=DEV)
    out, mean, rstd = scnn.layer_norm_fwd(x)
    assert out.shape == (0, 12) and mean.shape == (0,)
    dx, dgamma, dbeta = scnn.layer_norm_bwd(x, x, None, mean, rstd)
    assert dx.shape == (0, 12) and not dgamma.any() and not dbeta.any()


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("channels", [24, 1000, 9000])
def test_any_start_and_strides(dtype, channels):
    d = make(21, 50, channels, dtype)
    flat = torch.empty(50 * channels + 1, dtype=dtype, device=DEV)
    flat[1:] = d["x"].view(-1)
    want = scnn.layer_norm_fwd(d["x"], d["gamma"], d["beta"])
    out = (torch.empty(50 * channels + 1, dtype=dtype, device=DEV)[1:].view(50, channels), torch.empty(50, device=DEV),
           torch.empty(50, device=DEV))
    got = scnn.layer_norm_fwd(flat[1:].view(50, channels), d["gamma"], d["beta"], out=out)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = scnn.layer_norm_fwd(d["x"].t().contiguous().t(), d["gamma"].flip(0).flip(0), d["beta"])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    back = scnn.layer_norm_bwd(d["x"], d["g"], d["gamma"], *want[1:])
    other = scnn.layer_norm_bwd(flat[1:].view(50, channels), d["g"].t().contiguous().t(), d["gamma"], *want[1:])
    assert all(torch.equal(a, b) for a, b in zip(back, other))


def test_offsets_past_32_bits():
    rows, channels = 140001, 16000
    x = torch.zeros((rows, channels), dtype=torch.bfloat16, device=DEV)
    last = make(17, 40, channels, torch.bfloat16)
    x[-40:] = last["x"]
    assert x.numel() > 1 << 31
    out, mean, rstd = scnn.layer_norm_fwd(x, last["gamma"], last["beta"])
    want = scnn.layer_norm_fwd(last["x"], last["gamma"], last["beta"])
    for a, b in zip((out, mean, rstd), ref.layer_norm_fwd(last["x"], last["gamma"], last["beta"], 1e-5, torch.bfloat16)):
        ref.assert_within(a[-40:], b)
    g = out.zero_()
    g[-40:] = last["g"]
    back = scnn.layer_norm_bwd(x, g, last["gamma"], mean, rstd)
    for i, b in enumerate(ref.layer_norm_bwd(last["x"], last["g"], last["gamma"], want[1], want[2], torch.bfloat16)):
        ref.assert_within(back[i][-40:] if i == 0 else back[i], b)


def test_many_rows_of_every_shape():
    """Enough rows for the forms that long lists take: several vectors a lane or a thread."""
    for k, (rows, channels, dtype) in enumerate(((2100, 1500, torch.float32), (2100, 2000, torch.bfloat16), (2050, 3999, torch.float16),
                                                 (2050, 2047, torch.float32), (2050, 8000, torch.bfloat16), (2050, 4001, torch.float32))):
        d = make(40 + k, rows, channels, dtype)
        got = scnn.layer_norm_fwd(d["x"], d["gamma"], d["beta"])
        for a, b in zip(got, ref.layer_norm_fwd(d["x"], d["gamma"], d["beta"], 1e-5, dtype)):
            ref.assert_within(a, b)
        for a, b in zip(scnn.layer_norm_bwd(d["x"], d["g"], d["gamma"], got[1], got[2]),
                        ref.layer_norm_bwd(d["x"], d["g"], d["gamma"], got[1], got[2], dtype)):
            ref.assert_within(a, b)


def test_captured_and_replayed_and_another_stream():
    d = make(31, 500, 96, torch.float32)
    outs = (torch.empty((500, 96), device=DEV), torch.empty(500, device=DEV), torch.empty(500, device=DEV))
    grads = (torch.empty((500, 96), device=DEV), torch.empty(96, device=DEV), torch.empty(96, device=DEV))
    ws = torch.empty(scnn.layer_norm_bwd_workspace(torch.float32, 500, 96), dtype=torch.uint8, device=DEV)

    def step(stream=None):
        scnn.layer_norm_fwd(d["x"], d["gamma"], d["beta"], out=outs, stream=stream)
        scnn.layer_norm_bwd(d["x"], d["g"], d["gamma"], outs[1], outs[2], out=grads, workspace=ws, stream=stream)

    def eager():
        y, m, r = scnn.layer_norm_fwd(d["x"], d["gamma"], d["beta"])
        return (y, m, r, *scnn.layer_norm_bwd(d["x"], d["g"], d["gamma"], m, r))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*outs, *grads), eager()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        fresh = make(60 + k, 500, 96, torch.float32)
        for name in d:
            d[name].copy_(fresh[name])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*outs, *grads), eager()))
