"""Linear layers (forward and gradients) on the GPU against their formulas in 64 bits."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# (rows, c_in, c_out): one of everything, the few-row kernel and its end, tiles and their edges, odd widths, long sums
SIZES = [(1, 1, 1), (1, 1024, 40), (2, 7, 3), (3, 33, 17), (4, 64, 16), (5, 300, 19), (8, 100, 130), (9, 65, 63), (16, 16, 16),
         (64, 64, 64), (65, 129, 67), (200, 31, 257), (1000, 24, 40), (130, 1001, 505), (70, 4100, 33), (300, 256, 512), (3000, 1, 5),
         (257, 520, 264), (300, 8, 72), (40, 72, 8), (300, 56, 200), (5, 24, 16)]


def make(seed, rows, c_in, c_out, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, s=1.0):
        return (torch.randn(*shape, generator=g) * s).to(dtype).to(DEV)

    return {"x": normal(rows, c_in, s=scale).clamp_(min=-0.5 * scale), "w": normal(c_in, c_out, s=(2.0 / c_in) ** 0.5),
            "bias": normal(c_out, s=0.3), "residual": normal(rows, c_out), "g": normal(rows, c_out, s=0.5)}


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("k,size", list(enumerate(SIZES)), ids=str)
def test_forward_matches_the_formula(k, size, dtype):
    name = tuple(scnn.ACTIVATIONS)[k % 4]
    for bias, residual in ((False, False), (True, True), (True, False)):
        d = make(k, *size, dtype)
        b, r = d["bias"] if bias else None, d["residual"] if residual else None
        out, pre = scnn.linear_fwd(d["x"], d["w"], b, act=name, residual=r, keep_pre=True)
        want, want_pre = ref.linear_fwd(d["x"], d["w"], b, name, r, dtype)
        ref.assert_within(out, want, "out")
        ref.assert_within(pre, want_pre, "pre")
        again = scnn.linear_fwd(d["x"], d["w"], b, act=name, residual=r)
        assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("k,size", list(enumerate(SIZES)), ids=str)
def test_gradients_match_the_formula(k, size, dtype):
    name = tuple(scnn.ACTIVATIONS)[(k + 1) % 4]
    d = make(50 + k, *size, dtype)
    pre = ref.linear_fwd(d["x"], d["w"], d["bias"], "none", None, dtype)[1][0].to(dtype).to(DEV)
    got = scnn.linear_bwd(d["x"], d["w"], d["g"], act=name, pre=pre)
    want = ref.linear_bwd(d["x"], d["w"], d["g"], name, None if name == "none" else pre, dtype)
    for what, a, b in zip(("dx", "dw", "dbias"), got, want):
        ref.assert_within(a, b, what)
    for a, b in zip(scnn.linear_bwd(d["x"], d["w"], d["g"], act=name, pre=pre), got):
        assert torch.equal(a, b)
    for i in range(3):
        one = scnn.linear_bwd(d["x"], d["w"], d["g"], act=name, pre=pre, want=[i == j for j in range(3)])
        assert [o is None for o in one] == [i != j for j in range(3)] and torch.equal(one[i], got[i])


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("size", [(16392, 520, 520), (2000, 600, 1032), (1030, 2904, 2904), (30, 2056, 1000), (4100, 130, 1160)], ids=str)
def test_large_tiles(size, dtype):
    """Sizes that take every tile of every product, with rows, columns and k that end inside a tile."""
    d = make(7, *size, dtype)
    out, pre = scnn.linear_fwd(d["x"], d["w"], d["bias"], act="gelu", residual=d["residual"], keep_pre=True)
    want, want_pre = ref.linear_fwd(d["x"], d["w"], d["bias"], "gelu", d["residual"], dtype)
    ref.assert_within(out, want, "out")
    ref.assert_within(pre, want_pre, "pre")
    got = scnn.linear_bwd(d["x"], d["w"], d["g"], act="gelu", pre=pre)
    for what, a, b in zip(("dx", "dw", "dbias"), got, ref.linear_bwd(d["x"], d["w"], d["g"], "gelu", pre, dtype)):
        ref.assert_within(a, b, what)
    count = torch.tensor([size[0] - 13], dtype=torch.int64, device=DEV)
    n = size[0] - 13
    d["x"][n:] = float("nan")
    d["g"][n:] = float("nan")
    part = torch.full_like(out, 3.0)
    scnn.linear_fwd(d["x"], d["w"], d["bias"], act="gelu", residual=d["residual"], rows_dev=count, out=part)
    assert torch.equal(part[:n], out[:n]) and bool((part[n:] == 3).all())
    few = scnn.linear_bwd(d["x"], d["w"], d["g"], act="gelu", pre=pre, rows_dev=count)
    assert torch.equal(few[0][:n], got[0][:n])
    for what, a, b in zip(("dw", "dbias"), few[1:], ref.linear_bwd(d["x"][:n], d["w"], d["g"][:n], "gelu", pre[:n], dtype)[1:]):
        ref.assert_within(a, b, what)


@pytest.mark.parametrize("size", [(6, 50, 40), (150, 70, 90), (64, 3000, 20), (1000, 8, 8)], ids=str)
def test_whole_numbers_come_out_exactly(size):
    """Sums of small whole numbers are exact in fp32, whatever the order: every index is checked to the bit."""
    rows, c_in, c_out = size
    g = torch.Generator().manual_seed(rows)
    x, w, d = (torch.randint(-8, 9, s, generator=g).float() for s in ((rows, c_in), (c_in, c_out), (rows, c_out)))
    assert torch.equal(scnn.linear_fwd(x.to(DEV), w.to(DEV)).cpu(), x @ w)
    dx, dw, db = scnn.linear_bwd(x.to(DEV), w.to(DEV), d.to(DEV))
    assert torch.equal(dx.cpu(), d @ w.t()) and torch.equal(dw.cpu(), x.t() @ d) and torch.equal(db.cpu(), d.sum(0))


@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu"])
def test_gradients_match_differences(name):
    """Central differences of the 64-bit form, and the kernels' gradients against them."""
    d = {k: v.cpu().double() for k, v in make(3, 7, 6, 5, torch.float32).items()}

    def loss(x, w, b):
        return (ref.act(x @ w + b, name) * d["g"]).sum()

    pre = (d["x"] @ d["w"] + d["bias"]).float()
    got = scnn.linear_bwd(*(d[k].float().to(DEV) for k in ("x", "w", "g")), act=name, pre=pre.to(DEV))
    h = 1e-5
    for i, key in enumerate(("x", "w", "bias")):
        args = [d["x"], d["w"], d["bias"]]
        for at in range(args[i].numel()):
            e = torch.zeros_like(args[i]).view(-1)
            e[at] = h
            hi = [a + e.view_as(a) if j == i else a for j, a in enumerate(args)]
            lo = [a - e.view_as(a) if j == i else a for j, a in enumerate(args)]
            slope = (loss(*hi) - loss(*lo)) / (2 * h)
            # h^2 times third derivatives below 1, 64-bit cancellation, and fp32 sums of up to seven terms of size 3
            assert abs(float(got[i].view(-1)[at]) - float(slope)) < 1e-5, (key, at)


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("rows", [3, 40])
def test_infinities_nan_and_extremes(dtype, rows):
    """They reach the outputs that they stand behind, as the formula has it, and no others."""
    top, small = torch.finfo(dtype).max, torch.finfo(dtype).tiny
    d = make(9, rows, 70, 66, dtype)
    x, w = d["x"], d["w"]
    x[0, 5] = float("inf")
    x[1, 6] = float("nan")
    x[2, :] = small * 0.25                        # below the normal numbers
    w[:, 3] = 0
    w[7, 11] = float("-inf")
    w[9, 65] = float("nan")
    out = scnn.linear_fwd(x, w, d["bias"])
    ref.assert_within(out, ref.linear_fwd(x, w, d["bias"], "none", None, dtype)[0], "out")
    dx, dw, db = scnn.linear_bwd(x, w, d["g"])
    for a, b in zip((dx, dw, db), ref.linear_bwd(x, w, d["g"], "none", None, dtype)):
        ref.assert_within(a, b)
    if dtype == torch.float32:
        x = torch.full((rows, 64), 1e30, device=DEV)
        w = torch.full((64, 40), 1e-35, device=DEV)
        ref.assert_within(scnn.linear_fwd(x, w), ref.linear_fwd(x, w, None, "none", None, dtype)[0], "large by small")
        x = torch.full((rows, 2), top, device=DEV)
        x[:, 1] = -top
        w = torch.ones((2, 3), device=DEV)
        assert not scnn.linear_fwd(x, w).any()


@pytest.mark.parametrize("size", [(40, 64, 48), (3, 64, 48), (200, 96, 130), (300, 24, 24)], ids=str)
@pytest.mark.parametrize("power", [-104, -110, -120, -127])
def test_small_values_keep_their_bits(size, power):
    """Magnitudes around 2^-109, where three bf16 numbers begin not to hold an fp32 value: products with large ones."""
    d = make(13, *size, torch.float32)
    x, w = d["x"] * 2.0 ** power, d["w"] * 2.0 ** 100
    ref.assert_within(scnn.linear_fwd(x, w), ref.linear_fwd(x, w, None, "none", None, torch.float32)[0], "out")
    g = d["g"] * 2.0 ** power
    for a, b in zip(scnn.linear_bwd(x * 2.0 ** 50, w, g), ref.linear_bwd(x * 2.0 ** 50, w, g, "none", None, torch.float32)):
        ref.assert_within(a, b)


def test_offsets_past_32_bits():
    """More than 2^31 values in an array: the last rows are as a call on them alone gives them."""
    rows, width = 140001, 16400
    w = make(15, 4, 16, width, torch.bfloat16)["w"]
    x = torch.zeros((rows, 16), dtype=torch.bfloat16, device=DEV)
    last = make(16, 70, 16, width, torch.bfloat16)
    x[-70:] = last["x"]
    out = scnn.linear_fwd(x, w, act="relu")
    assert out.numel() > 1 << 31
    # (another tile may add another order of sixteen products: one rounding of the result)
    want = ref.linear_fwd(last["x"], w, None, "relu", None, torch.bfloat16)[0]
    ref.assert_within(out[-70:], want)
    assert not out[:1000].any()
    g = torch.zeros_like(out)
    g[-70:] = last["g"]
    del out
    dx, dw, db = scnn.linear_bwd(x, w, g)
    del g
    for a, b in zip((dx[-70:], dw, db), ref.linear_bwd(last["x"], w, last["g"], "none", None, torch.bfloat16)):
        ref.assert_within(a, b)
    assert not dx[:-70].any()


@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
def test_activations_of_far_values(name):
    z = torch.tensor([[0.0, -0.0, 1e-30, -1e-30, 20.0, -20.0, 100.0, -100.0, float("nan"), float("inf")]], device=DEV)
    eye = torch.eye(10, device=DEV)
    out, pre = scnn.linear_fwd(torch.zeros((1, 10), device=DEV), eye, z[0].contiguous(), act=name, keep_pre=True)
    want = ref.act(z.double().cpu(), name)
    if name == "silu":
        want[0, 9] = float("inf")
    got = out.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and float(got[0, 9]) == float("inf")
    ok = torch.isfinite(want)
    assert ((got - want).abs()[ok] <= 32 * ref.U32 * want.abs()[ok] + 1e-37).all(), (got, want)
    g = torch.ones((1, 10), device=DEV)
    slope = scnn.linear_bwd(torch.zeros((1, 10), device=DEV), eye, g, act=name, pre=pre)[2].double().cpu()
    ws = ref.act_slope(z.double().cpu(), name)[0]
    assert ((slope - ws).abs()[:8] <= 32 * ref.U32 * (1 + z.cpu().abs()[0, :8])).all(), (slope, ws)


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
@pytest.mark.parametrize("cap,count", [(100, 37), (100, 0), (100, -5), (100, 100), (100, 1 << 40), (6, 2), (6, 0), (700, 129)])
def test_row_count_from_the_device(cap, count, dtype):
    """Rows past the count hold NaN: nothing of them is read, and what lies behind the last row stays."""
    n = max(0, min(cap, count))
    d = make(11, cap, 40, 72, dtype)
    pre = make(12, cap, 40, 72, dtype)["residual"]
    for t in (d["x"], d["g"], d["residual"], pre):
        t[n:] = float("nan")
    rows_dev = torch.tensor([count, 7], dtype=torch.int64, device=DEV)
    out, keep = torch.full((cap, 72), 7.0, dtype=dtype, device=DEV), torch.full((cap, 72), 8.0, dtype=dtype, device=DEV)
    scnn.linear_fwd(d["x"], d["w"], d["bias"], act="gelu", residual=d["residual"], rows_dev=rows_dev, out=out, pre=keep)
    assert bool((out[n:] == 7).all()) and bool((keep[n:] == 8).all())
    want, want_pre = ref.linear_fwd(d["x"][:n], d["w"], d["bias"], "gelu", d["residual"][:n], dtype)
    ref.assert_within(out[:n], want)
    ref.assert_within(keep[:n], want_pre)
    for name in ("none", "silu"):
        dx = torch.full((cap, 40), 7.0, dtype=dtype, device=DEV)
        dw, db = torch.empty((40, 72), dtype=dtype, device=DEV), torch.empty(72, dtype=dtype, device=DEV)
        scnn.linear_bwd(d["x"], d["w"], d["g"], act=name, pre=pre, rows_dev=rows_dev, out=(dx, dw, db))
        assert bool((dx[n:] == 7).all())
        for a, b in zip((dx[:n], dw, db), ref.linear_bwd(d["x"][:n], d["w"], d["g"][:n], name,
                                                          None if name == "none" else pre[:n], dtype)):
            ref.assert_within(a, b, name)


def test_longest_sums():
    """More k than the few-row kernel splits over the card."""
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn((1, 20000003), generator=g).to(DEV), torch.randn((20000003, 1), generator=g).to(DEV)
    ref.assert_within(scnn.linear_fwd(x, w), ref.linear_fwd(x, w, None, "none", None, torch.float32)[0])
    assert torch.equal(scnn.linear_fwd(x, w), scnn.linear_fwd(x, w))


@pytest.mark.parametrize("size", [(200, 40, 24), (200, 20, 24), (130, 200, 100)], ids=str)
@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
def test_null_operands_of_what_is_not_asked_for(size, dtype):
    """Through the C ABI: no x without dw, no w without dx."""
    L = scnn.load_library()
    rows, c_in, c_out = size
    d = make(71, *size, dtype)
    want = ref.linear_bwd(d["x"], d["w"], d["g"], "none", None, dtype)
    code = scnn.DTYPES[dtype]
    ws = torch.empty(scnn.linear_bwd_workspace(dtype, *size), dtype=torch.uint8, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    outs = [torch.empty_like(d["x"]), torch.empty_like(d["w"]), torch.empty(c_out, dtype=dtype, device=DEV)]
    for ask in ((True, False, True), (False, True, True), (False, False, True), (True, False, False), (False, True, False)):
        p = [o.data_ptr() if a else None for o, a in zip(outs, ask)]
        rc = L.linear_bwd(code, d["x"].data_ptr() if ask[1] else None, rows, None, c_in, d["w"].data_ptr() if ask[0] else None,
                          c_out, 0, None, d["g"].data_ptr(), *p, ws.data_ptr(), ws.numel(), stream)
        assert rc == 0
        for o, a, b in zip(outs, ask, want):
            if a:
                ref.assert_within(o, b, str(ask))
            o.fill_(float("nan"))


def test_no_rows():
    x, w = torch.empty((0, 5), device=DEV), torch.ones((5, 3), device=DEV)
    assert scnn.linear_fwd(x, w).shape == (0, 3)
    dx, dw, db = scnn.linear_bwd(x, w, torch.empty((0, 3), device=DEV), act="relu", pre=torch.empty((0, 3), device=DEV))
    assert dx.shape == (0, 5) and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", ref.TYPES, ids=str)
def test_any_start_and_strides(dtype):
    """Arrays that start one element into their storage, transposed and strided inputs, results in arrays of the caller."""
    rows, c_in, c_out = 90, 64, 72
    d = make(21, rows, c_in, c_out, dtype)

    def moved(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
        flat[1:] = t.reshape(-1)
        return flat[1:].view(t.shape)

    want = scnn.linear_fwd(d["x"], d["w"], d["bias"], act="gelu", residual=d["residual"])
    out = moved(torch.zeros_like(want))
    got = scnn.linear_fwd(moved(d["x"]), moved(d["w"]), moved(d["bias"]), act="gelu", residual=moved(d["residual"]), out=out)
    assert got is out
    exact, _ = ref.linear_fwd(d["x"], d["w"], d["bias"], "gelu", d["residual"], dtype)
    ref.assert_within(got, exact)
    wide = torch.empty((rows, 2 * c_in), dtype=dtype, device=DEV)
    wide[:, ::2] = d["x"]
    assert torch.equal(scnn.linear_fwd(wide[:, ::2], d["w"].t().contiguous().t(), d["bias"], act="gelu", residual=d["residual"]), want)
    assert torch.equal(scnn.linear_fwd(d["x"], d["w"], d["bias"].new_full((1,), 0.5).expand(c_out)),
                       scnn.linear_fwd(d["x"], d["w"], torch.full_like(d["bias"], 0.5)))
    back = scnn.linear_bwd(d["x"], d["w"], d["g"])
    other = scnn.linear_bwd(moved(d["x"]), moved(d["w"]), moved(d["g"]), out=tuple(moved(b) for b in back))
    for a, b in zip(other, ref.linear_bwd(d["x"], d["w"], d["g"], "none", None, dtype)):
        ref.assert_within(a, b)
    summed = d["residual"].clone()
    scnn.linear_fwd(d["x"], d["w"], d["bias"], act="gelu", residual=summed, out=summed)
    assert torch.equal(summed, want)


def test_refusals_of_tensors():
    d = make(23, 10, 16, 24, torch.float32)
    x, w, b, r, g = d["x"], d["w"], d["bias"], d["residual"], d["g"]
    for bad in (lambda: scnn.linear_fwd(x, w.t()), lambda: scnn.linear_fwd(x, w.half()), lambda: scnn.linear_fwd(x, w, b[:-1]),
                lambda: scnn.linear_fwd(x, w, residual=r[:-1]), lambda: scnn.linear_fwd(x, w, act="tanh"),
                lambda: scnn.linear_fwd(x.double(), w.double()), lambda: scnn.linear_fwd(x, w.cpu()),
                lambda: scnn.linear_fwd(x, w, out=torch.empty((24, 10), device=DEV).t()),
                lambda: scnn.linear_fwd(x, w, rows_dev=torch.ones(1, device=DEV)), lambda: scnn.linear_fwd(x[0], w),
                lambda: scnn.linear_bwd(x, w, g, act="relu"), lambda: scnn.linear_bwd(x, w, g[:, :-1])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(scnn.ScnnError):   # in place on an input that is still read
        scnn.linear_fwd(x, torch.eye(16, device=DEV), out=x)
    with pytest.raises(scnn.ScnnError):
        scnn.linear_bwd(x, w, g, out=(x, torch.empty_like(w), torch.empty_like(b)))


def test_another_stream_and_two_at_once():
    sizes = ((300, 500, 260), (5, 900, 300))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    data = [make(31 + i, *s, torch.float32) for i, s in enumerate(sizes)]
    want = [scnn.linear_fwd(d["x"], d["w"], d["bias"]) for d in data]
    back = [scnn.linear_bwd(d["x"], d["w"], d["g"]) for d in data]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, d in zip(streams, data):
            got.append((scnn.linear_fwd(d["x"], d["w"], d["bias"], stream=s), scnn.linear_bwd(d["x"], d["w"], d["g"], stream=s)))
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(got):
        assert torch.equal(a, want[i % 2])
        assert all(torch.equal(p, q) for p, q in zip(b, back[i % 2]))


def test_captured_without_an_eager_run_before():
    """The large tiles' shared memory is asked for by the call itself, in a capture too."""
    d = make(43, 1000, 4096, 16640, torch.float16)
    out = torch.empty((1000, 16640), dtype=torch.float16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        scnn.linear_fwd(d["x"], d["w"], d["bias"], out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, scnn.linear_fwd(d["x"], d["w"], d["bias"]))


def test_captured_and_replayed():
    d = make(41, 64, 2000, 96, torch.float32)
    out, pre = torch.empty((64, 96), device=DEV), torch.empty((64, 96), device=DEV)
    grads = (torch.empty((64, 2000), device=DEV), torch.empty((2000, 96), device=DEV), torch.empty(96, device=DEV))
    ws = torch.empty(scnn.linear_fwd_workspace(torch.float32, 64, 2000, 96), dtype=torch.uint8, device=DEV)
    wb = torch.empty(scnn.linear_bwd_workspace(torch.float32, 64, 2000, 96, "gelu"), dtype=torch.uint8, device=DEV)

    def step():
        scnn.linear_fwd(d["x"], d["w"], d["bias"], act="gelu", out=out, pre=pre, workspace=ws)
        scnn.linear_bwd(d["x"], d["w"], d["g"], act="gelu", pre=pre, out=grads, workspace=wb)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        fresh = make(60 + k, 64, 2000, 96, torch.float32)
        for name in ("x", "w", "bias", "g"):
            d[name].copy_(fresh[name])
        graph.replay()
        torch.cuda.synchronize()
        y, z = scnn.linear_fwd(fresh["x"], fresh["w"], fresh["bias"], act="gelu", keep_pre=True)
        eager = scnn.linear_bwd(fresh["x"], fresh["w"], fresh["g"], act="gelu", pre=z)
        assert torch.equal(out, y) and torch.equal(pre, z)
        assert all(torch.equal(a, b) for a, b in zip(grads, eager))
