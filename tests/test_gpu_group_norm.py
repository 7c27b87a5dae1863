"""Group norm with its activation (forward and gradients) and sample_offsets on the GPU against their formulas in 64 bits."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from . import block_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ACTS = ("none", "relu", "gelu", "silu")
TYPES = (torch.float32, torch.bfloat16, torch.float16)
# (rows, channels, groups, offsets or number of equal samples): one value, one row, odd widths, groups of one channel and one
# group, vectors that hold several groups, empty samples first, last and in between, a row before and behind the samples,
# samples that end inside a block, wide rows, rows past a workgroup's columns, groups past them
CASES = [(1, 1, 1, 1), (1, 24, 8, 1), (512, 24, 8, 1), (7, 3, 3, [0, 7]), (300, 5, 1, [0, 0, 100, 100, 299, 300, 300]),
         (64, 8, 8, 4), (1000, 25, 5, [0, 1, 2, 900, 1000]), (1000, 25, 5, [3, 400, 990]), (50, 40, 10, [0, 0, 0]),
         (4000, 16, 4, [0, 1000, 1001, 3999, 4000]), (20000, 24, 6, [0, 7777, 20000]), (9001, 19, 19, [0, 9001]),
         (5000, 35, 7, [11, 2500, 2500, 4900]), (3000, 64, 8, 6), (6000, 7, 1, 3), (257, 33, 11, [0, 100, 257]),
         (40, 1000, 8, [0, 13, 40]), (300, 1001, 7, [0, 150, 300]), (90, 2048, 32, 3), (33, 2056, 2056, [0, 33]),
         (64, 4096, 1, 2), (25, 4100, 4, [0, 10, 25]), (40, 5000, 5, 1), (30, 9000, 3000, [0, 7, 30]), (12, 20000, 2, [0, 5, 12]),
         (9, 17001, 3, 1), (70000, 2, 2, [0, 30000, 70000]), (30011, 1, 1, [0, 5, 30000])]


def make(seed, rows, channels, dtype, shift=0.5):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, s=1.0, m=0.0):
        return (torch.randn(*shape, generator=g) * s + m).to(dtype).to(DEV)

    return {"x": normal(rows, channels, s=1.5, m=shift), "gamma": normal(channels, s=0.2, m=1.0), "beta": normal(channels, s=0.3),
            "g": normal(rows, channels, s=0.5)}


def where(offsets):
    if isinstance(offsets, int):
        return {"batch": offsets}, {}
    t = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    return {"offsets": t}, {"offsets": t}


def check(d, case, act, gamma, beta, dtype, eps=1e-5):
    rows, channels, groups, offsets = case
    fwd, bwd = where(offsets)
    batch = offsets if isinstance(offsets, int) else len(offsets) - 1
    samples = ref.bounds_of(None if isinstance(offsets, int) else offsets, rows, batch)
    lo, hi = samples[0][0], samples[-1][1]
    outs = (torch.full((rows, channels), 7.0, dtype=dtype, device=DEV), torch.empty((batch, groups), device=DEV),
            torch.empty((batch, groups), device=DEV))
    out, mean, rstd = scnn.group_norm_fwd(d["x"], groups, gamma, beta, eps=eps, act=act, out=outs, **fwd)
    assert bool((out[:lo] == 7).all()) and bool((out[hi:] == 7).all())
    for what, a, b in zip(("out", "mean", "rstd"), (out[lo:hi], mean, rstd),
                          ref.group_norm_fwd(d["x"], groups, gamma, beta, samples, eps, act, dtype)):
        ref.assert_within(a, b, what)
    grads = (torch.full((rows, channels), 7.0, dtype=dtype, device=DEV), torch.empty(channels, dtype=dtype, device=DEV),
             torch.empty(channels, dtype=dtype, device=DEV))
    back = scnn.group_norm_bwd(d["x"], d["g"], groups, gamma, beta, mean, rstd, act=act, out=grads, **bwd)
    assert bool((back[0][:lo] == 7).all()) and bool((back[0][hi:] == 7).all())
    want = ref.group_norm_bwd(d["x"], d["g"], groups, gamma, beta, mean, rstd, samples, act, dtype)
    for what, a, b in zip(("dx", "dgamma", "dbeta"), (back[0][lo:hi], *back[1:]), want):
        ref.assert_within(a, b, what)
    return outs, back, fwd, bwd


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("k,case", list(enumerate(CASES)), ids=str)
def test_matches_the_formulas(k, case, dtype):
    rows, channels, groups, _ = case
    d = make(k, rows, channels, dtype)
    act = ACTS[k % 4]
    outs, back, fwd, bwd = check(d, case, act, d["gamma"], d["beta"], dtype)
    again = scnn.group_norm_fwd(d["x"], groups, d["gamma"], d["beta"], act=act, **fwd)
    assert torch.equal(again[1], outs[1]) and torch.equal(again[2], outs[2])
    for i in range(3):
        one = scnn.group_norm_bwd(d["x"], d["g"], groups, d["gamma"], d["beta"], *outs[1:], act=act,
                                  want=[i == j for j in range(3)], **bwd)
        assert [o is None for o in one] == [i != j for j in range(3)]
        if i:
            assert torch.equal(one[i], back[i])
        else:
            lo, hi = (0, rows) if "batch" in fwd else (int(fwd["offsets"][0]), int(fwd["offsets"][-1]))
            assert torch.equal(one[0][lo:hi], back[0][lo:hi])


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("case", [(700, 24, 6, [0, 300, 700]), (20000, 25, 5, [0, 9000, 20000]), (60, 4100, 2, [0, 25, 60])], ids=str)
def test_activations_and_what_is_left_out(case, act):
    for dtype in TYPES:
        d = make(3, case[0], case[1], dtype)
        check(d, case, act, None, None, dtype)
        check(d, case, act, d["gamma"], None, dtype)
        check(d, case, act, None, d["beta"], dtype, eps=0.1)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("case", [(4000, 517, 11, [0, 7, 2500, 4000]), (30, 2051, 2051, 1), (30, 1027, 1027, [0, 11, 29]), (700, 4099, 1, 1),
                                  (600, 6150, 3, [1, 50, 599]), (1500, 1999, 1, 3), (2500, 1026, 9, 5), (90, 2050, 1025, 1)], ids=str)
def test_rows_that_end_inside_a_vector(case, dtype):
    """Of one group and many, of several slabs, the last narrower than a vector, and of groups in pieces; a NaN stays in its group."""
    rows, channels, groups, offsets = case
    d = make(41, rows, channels, dtype)
    check(d, case, "silu", d["gamma"], d["beta"], dtype)
    row = offsets[1] - 1 if not isinstance(offsets, int) else rows - 1
    fwd, bwd = where(offsets)
    if groups > 1:
        per = channels // groups
        for j in (0, groups - 2, groups - 1):
            x = d["x"].clone()
            x[row, (j + 1) * per - 1] = float("nan")
            out, mean, rstd = scnn.group_norm_fwd(x, groups, d["gamma"], d["beta"], **fwd)
            bad = torch.zeros(groups, dtype=torch.bool, device=DEV)
            bad[j] = True
            b = 0 if not isinstance(offsets, int) else offsets - 1
            assert torch.equal(mean[b].isnan(), bad) and torch.equal(out[row].isnan(), bad.repeat_interleave(per))
            dx, dgamma, _ = scnn.group_norm_bwd(x, d["g"], groups, d["gamma"], d["beta"], mean, rstd, **bwd)
            assert torch.equal(dx[row].isnan(), bad.repeat_interleave(per)) and torch.equal(dgamma.isnan(), bad.repeat_interleave(per))


def test_gradients_match_differences():
    rows, channels, groups, samples = 7, 6, 3, [(0, 3), (3, 7)]
    d = {k: v.cpu().double() for k, v in make(3, rows, channels, torch.float32).items()}

    def loss(x, gamma, beta, name):
        total = 0
        for a, b in samples:
            v = x[a:b].view(b - a, groups, 2)
            m = v.mean((0, 2), keepdim=True)
            s = ((v - m) ** 2).mean((0, 2), keepdim=True)
            z = ((v - m) / torch.sqrt(s + 1e-5)).view(b - a, channels) * gamma + beta
            total = total + (ref.act(z, name) * d["g"][a:b]).sum()
        return total

    f = {k: v.float().to(DEV) for k, v in d.items()}
    offsets = torch.tensor([0, 3, 7], device=DEV)
    for name in ("none", "gelu", "silu"):
        _, mean, rstd = scnn.group_norm_fwd(f["x"], groups, f["gamma"], f["beta"], offsets=offsets, act=name)
        got = scnn.group_norm_bwd(f["x"], f["g"], groups, f["gamma"], f["beta"], mean, rstd, offsets=offsets, act=name)
        h = 1e-5
        for i in range(3):
            args = [d["x"], d["gamma"], d["beta"]]
            for at in range(args[i].numel()):
                e = torch.zeros_like(args[i]).view(-1)
                e[at] = h
                hi = [a + e.view_as(a) if j == i else a for j, a in enumerate(args)]
                lo = [a - e.view_as(a) if j == i else a for j, a in enumerate(args)]
                slope = (loss(*hi, name) - loss(*lo, name)) / (2 * h)
                # 64-bit cancellation over h, h^2 times third derivatives below 100, and some tens of fp32 roundings of size 3
                assert abs(float(got[i].view(-1)[at]) - float(slope)) < 2e-5, (name, i, at)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,channels,groups", [(40, 12, 3), (9000, 40, 4), (30, 9000, 2)])
def test_equal_values_and_values_far_from_zero(rows, channels, groups, dtype):
    x = torch.full((rows, channels), 3.0, dtype=dtype, device=DEV)
    x[rows // 2:] = torch.finfo(dtype).max / 64
    offsets = torch.tensor([0, rows // 2, rows], device=DEV)
    out, mean, rstd = scnn.group_norm_fwd(x, groups, offsets=offsets, eps=1e-3)
    assert not out.any() and bool((mean[0] == 3).all()) and bool((mean[1] == float(x[-1, 0])).all())
    assert torch.allclose(rstd.cpu(), torch.full((2, groups), 1e-3 ** -0.5))
    if dtype == torch.float32:
        d = make(5, rows, channels, dtype, shift=10000.0)
        d["x"][0, 0] = -1e6  # (the value that the sums are taken about, far from all others)
        check(d, (rows, channels, groups, [0, rows // 2, rows]), "none", None, None, dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,channels,groups", [(60, 20, 5), (20000, 24, 4), (30, 9000, 3)])
def test_nan_and_infinities_stay_in_their_groups(rows, channels, groups, dtype):
    d = make(7, rows, channels, dtype)
    cut, per = rows // 3, channels // groups
    offsets = torch.tensor([0, cut, rows], device=DEV)
    fwd = lambda: scnn.group_norm_fwd(d["x"], groups, d["gamma"], d["beta"], offsets=offsets, act="silu")  # noqa: E731
    clean = fwd()[0]
    for value, at in ((float("nan"), (1, per)), (float("inf"), (cut, 0)), (float("-inf"), (rows - 1, channels - 1))):
        kept = d["x"][at].clone()
        d["x"][at] = value
        out, mean, rstd = fwd()
        b, j = int(at[0] >= cut), at[1] // per
        hit = torch.zeros(rows, channels, dtype=torch.bool, device=DEV)
        hit[(0, cut)[b]:(cut, rows)[b], j * per:(j + 1) * per] = True
        assert bool(torch.isnan(out[hit]).all()) and torch.equal(out[~hit], clean[~hit])
        dx, dgamma, dbeta = scnn.group_norm_bwd(d["x"], d["g"], groups, d["gamma"], d["beta"], mean, rstd, offsets=offsets, act="silu")
        assert bool(torch.isnan(dx[hit]).all()) and bool(torch.isfinite(dx[~hit]).all())
        assert torch.equal(torch.isnan(dgamma), hit.any(0)) and torch.equal(torch.isnan(dbeta), hit.any(0))
        d["x"][at] = kept


def test_rows_outside_the_samples_are_not_read():
    for dtype in TYPES:
        for rows, channels, groups in ((100, 16, 4), (12000, 24, 4)):
            d = make(9, rows, channels, dtype)
            lo, hi = 5, rows - 7
            offsets = torch.tensor([lo, rows // 2, hi], device=DEV)
            for k in ("x", "g"):
                d[k][:lo] = float("nan")
                d[k][hi:] = float("nan")
            check(d, (rows, channels, groups, [lo, rows // 2, hi]), "gelu", d["gamma"], d["beta"], dtype)
            assert offsets.shape == (3,)


def test_numbers_outside_the_array_count_as_its_ends():
    rows, channels = 600, 16
    d = make(11, rows, channels, torch.float32)
    check(d, (rows, channels, 4, [-5, 200, 1 << 40]), "relu", d["gamma"], d["beta"], torch.float32)
    # numbers that do not ascend: no defined result, but an end to the call, and rows outside all of them stay
    for bad in ([300, 100, 400], [1 << 50, -(1 << 50), 7], [0, 600, 0, 600, 0]):
        t = torch.tensor(bad, device=DEV)
        out, mean, rstd = scnn.group_norm_fwd(d["x"], 4, d["gamma"], d["beta"], offsets=t)
        scnn.group_norm_bwd(d["x"], d["g"], 4, d["gamma"], d["beta"], mean, rstd, offsets=t)
    torch.cuda.synchronize()


def test_no_rows():
    x = torch.empty((0, 12), device=DEV)
    for kw in ({"batch": 3}, {"offsets": torch.zeros(4, dtype=torch.int64, device=DEV)}):
        out, mean, rstd = scnn.group_norm_fwd(x, 4, **kw)
        assert out.shape == (0, 12) and mean.shape == (3, 4) and not mean.any() and not rstd.any()
        dx, dgamma, dbeta = scnn.group_norm_bwd(x, x, 4, None, None, mean, rstd, offsets=kw.get("offsets"))
        assert dx.shape == (0, 12) and not dgamma.any() and not dbeta.any()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,channels", [(50, 24), (9000, 25), (9000, 40), (50, 9000)])
def test_any_start_and_strides(rows, channels, dtype):
    d = make(21, rows, channels, dtype)
    groups, offsets = 5 if channels % 5 == 0 else 4, torch.tensor([0, rows // 3, rows], device=DEV)
    want = scnn.group_norm_fwd(d["x"], groups, d["gamma"], d["beta"], offsets=offsets)
    flat = torch.empty(rows * channels + 1, dtype=dtype, device=DEV)
    flat[1:] = d["x"].view(-1)
    out = (torch.empty(rows * channels + 1, dtype=dtype, device=DEV)[1:].view(rows, channels), torch.empty(2, groups, device=DEV),
           torch.empty(2, groups, device=DEV))
    got = scnn.group_norm_fwd(flat[1:].view(rows, channels), groups, d["gamma"], d["beta"], offsets=offsets, out=out)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    wide = torch.stack([offsets, offsets], 1).view(-1)[::2]
    got = scnn.group_norm_fwd(d["x"].t().contiguous().t(), groups, d["gamma"].flip(0).flip(0), d["beta"], offsets=wide)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    back = scnn.group_norm_bwd(d["x"], d["g"], groups, d["gamma"], d["beta"], *want[1:], offsets=offsets)
    other = scnn.group_norm_bwd(flat[1:].view(rows, channels), d["g"].t().contiguous().t(), groups, d["gamma"], d["beta"],
                                *want[1:], offsets=offsets)
    assert all(torch.equal(a, b) for a, b in zip(back, other))


def test_offsets_past_32_bits():
    rows, channels = 140001, 16000
    x = torch.zeros((rows, channels), dtype=torch.bfloat16, device=DEV)
    last = make(17, 40, channels, torch.bfloat16)
    x[-40:] = last["x"]
    offsets = torch.tensor([0, rows - 40, rows], device=DEV)
    out, mean, rstd = scnn.group_norm_fwd(x, 10, last["gamma"], last["beta"], offsets=offsets)
    for a, b in zip((out[-40:], mean[1:], rstd[1:]),
                    ref.group_norm_fwd(last["x"], 10, last["gamma"], last["beta"], [(0, 40)], 1e-5, "none", torch.bfloat16)):
        ref.assert_within(a, b)
    g = out.zero_()
    g[-40:] = last["g"]
    back = scnn.group_norm_bwd(x, g, 10, last["gamma"], last["beta"], mean, rstd, offsets=offsets)
    want = ref.group_norm_bwd(last["x"], last["g"], 10, last["gamma"], last["beta"], mean[1:], rstd[1:], [(0, 40)], "none", torch.bfloat16)
    for i, b in enumerate(want):
        ref.assert_within(back[i][-40:] if i == 0 else back[i], b)


@pytest.mark.parametrize("rows,batch", [(3000, 700), (500, 5000), (20000, 65)])
def test_many_samples(rows, batch):
    g = torch.Generator().manual_seed(rows)
    cuts = sorted(torch.randint(0, rows + 1, (batch - 1,), generator=g).tolist())
    for channels, groups in ((6, 2), (40, 40)):
        d = make(23, rows, channels, torch.float32)
        check(d, (rows, channels, groups, [0] + cuts + [rows]), "silu", d["gamma"], d["beta"], torch.float32)


@pytest.mark.parametrize("size", [(400, 24, 6), (30000, 25, 5)], ids=str)
def test_captured_and_replayed_and_another_stream(size):
    rows, channels, groups = size
    d = make(31, rows, channels, torch.float32)
    offsets = torch.tensor([0, rows // 4, rows], device=DEV)
    outs = (torch.empty((rows, channels), device=DEV), torch.empty((2, groups), device=DEV), torch.empty((2, groups), device=DEV))
    grads = (torch.empty((rows, channels), device=DEV), torch.empty(channels, device=DEV), torch.empty(channels, device=DEV))
    room = [torch.empty(q(torch.float32, rows, 2, channels, groups), dtype=torch.uint8, device=DEV)
            for q in (scnn.group_norm_fwd_workspace, scnn.group_norm_bwd_workspace)]

    def step(stream=None):
        scnn.group_norm_fwd(d["x"], groups, d["gamma"], d["beta"], offsets=offsets, act="gelu", out=outs, workspace=room[0], stream=stream)
        scnn.group_norm_bwd(d["x"], d["g"], groups, d["gamma"], d["beta"], outs[1], outs[2], offsets=offsets, act="gelu", out=grads,
                            workspace=room[1], stream=stream)

    def eager():
        y, m, r = scnn.group_norm_fwd(d["x"], groups, d["gamma"], d["beta"], offsets=offsets, act="gelu")
        return (y, m, r, *scnn.group_norm_bwd(d["x"], d["g"], groups, d["gamma"], d["beta"], m, r, offsets=offsets, act="gelu"))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*outs, *grads), eager()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        fresh = make(60 + k, rows, channels, torch.float32)
        for name in d:
            d[name].copy_(fresh[name])
        offsets.copy_(torch.tensor([0, rows // (2 + k), rows]))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*outs, *grads), eager()))


def test_sample_offsets():
    g = torch.Generator().manual_seed(5)
    for rows, batch, ndim in ((0, 3, 2), (1, 1, 3), (10, 4, 3), (64, 64, 2), (65, 7, 3), (5000, 9, 2), (300000, 40, 3), (100, 1000, 3)):
        sample = torch.randint(0, batch, (rows,), generator=g).sort()[0]
        coords = torch.randint(0, 30, (rows, 1 + ndim), generator=g)
        coords[:, 0] = sample
        c = coords.to(torch.int32).to(DEV)
        want = torch.searchsorted(sample, torch.arange(batch + 1))
        assert torch.equal(scnn.sample_offsets(c, batch).cpu(), want)
        for count in (rows // 2, -4, 1 << 40):
            n = max(0, min(rows, count))
            out = torch.empty(batch + 1, dtype=torch.int64, device=DEV)
            scnn.sample_offsets(c, batch, rows_dev=torch.tensor([count], device=DEV), out=out)
            assert torch.equal(out.cpu(), torch.searchsorted(sample[:n], torch.arange(batch + 1)))
