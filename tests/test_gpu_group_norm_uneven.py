"""Group norm over samples of very unequal sizes: long ones beside many short and empty ones, whose work is divided on the device."""
import statistics

import pytest
import torch

import paper_1801_10585_amd as scnn
from . import block_ref as ref
from .test_gpu_group_norm import check, make
from .test_gpu_group_norm_sums import one_long

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def sizes(*runs):
    """Bounds from (number of samples, rows of each)."""
    cuts = [0]
    for count, rows in runs:
        for _ in range(count):
            cuts.append(cuts[-1] + rows)
    return cuts


def shifted(cuts, by):
    return [c + by for c in cuts]


# (rows, channels, groups, offsets), more than 131072 values and up to 32768 a sample on the average: one sample with nearly all rows,
# first, last and in between; two and three long ones next to each other, apart, and ending in the middle of a block; samples just below and
# above 65536 values; rows before the first and behind the last; odd rows, many groups, a batch of more samples than a wave has lanes
CASES = [(131072, 16, 4, one_long(131072, 64)), (9000, 64, 8, sizes((1, 8940), (60, 1))), (9000, 64, 8, sizes((60, 1), (1, 8940))),
         (20000, 25, 5, sizes((9, 11), (1, 7000), (1, 6901), (5, 0), (1, 3000), (40, 75))),
         (30000, 24, 6, sizes((3, 1), (1, 14001), (1, 2), (1, 15990), (30, 0), (4, 1))),
         (6200, 64, 8, sizes((1, 1023), (1, 1024), (1, 1025), (1, 1026), (1, 2047), (55, 1))),
         (9050, 64, 32, shifted(one_long(9000, 20), 17)), (3000, 300, 100, one_long(2990, 40)), (70000, 7, 7, one_long(70000, 33)),
         (4000, 200, 200, sizes((2, 0), (1, 2000), (100, 1), (1, 1900))), (150000, 3, 1, shifted(one_long(149990, 200), 3)),
         (1500, 510, 2, sizes((20, 5), (1, 1400)))]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("k", range(len(CASES)))
def test_matches_the_formulas(k, dtype):
    rows, channels, groups, offsets = case = CASES[k]
    assert rows * channels > 131072 and offsets == sorted(offsets) and offsets[-1] <= rows
    d = make(100 + k, rows, channels, dtype)
    act = ("silu", "none", "gelu", "relu")[k % 4]
    outs, back, fwd, bwd = check(d, case, act, d["gamma"], d["beta"], dtype)
    again = scnn.group_norm_fwd(d["x"], groups, d["gamma"], d["beta"], act=act, **fwd)
    lo, hi = offsets[0], offsets[-1]
    assert torch.equal(again[0][lo:hi], outs[0][lo:hi]) and torch.equal(again[1], outs[1]) and torch.equal(again[2], outs[2])
    only = scnn.group_norm_bwd(d["x"], d["g"], groups, d["gamma"], d["beta"], *outs[1:], act=act, want=(True, False, False), **bwd)
    assert torch.equal(only[0][lo:hi], back[0][lo:hi])
    only = scnn.group_norm_bwd(d["x"], d["g"], groups, d["gamma"], d["beta"], *outs[1:], act=act, want=(False, True, True), **bwd)
    assert torch.equal(only[1], back[1]) and torch.equal(only[2], back[2])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("k", range(len(CASES)))
def test_sums_of_whole_numbers_to_the_last_bit(k, dtype):
    rows, channels, groups, offsets = CASES[k]
    gen = torch.Generator().manual_seed(k)
    x, g = (torch.randint(-8, 9, (rows, channels), generator=gen).to(dtype) for _ in range(2))
    for t in (x, g):  # (outside the samples: not read)
        t[:offsets[0]] = float("nan")
        t[offsets[-1]:] = float("nan")
    a, b = x[offsets[0]:offsets[-1]].double(), g[offsets[0]:offsets[-1]].double()
    mean, rstd = torch.zeros(len(offsets) - 1, groups, device=DEV), torch.ones(len(offsets) - 1, groups, device=DEV)
    where = torch.tensor(offsets, device=DEV)
    for wanted in ((True, True, True), (False, True, True)):
        got = scnn.group_norm_bwd(x.to(DEV), g.to(DEV), groups, None, None, mean, rstd, offsets=where, want=wanted)
        assert torch.equal(got[1].cpu(), (a * b).sum(0).float().to(dtype)) and torch.equal(got[2].cpu(), b.sum(0).float().to(dtype))


def test_blocks_of_more_rows_than_a_workgroup_keeps():
    """2^26 values: a block is 8192 rows, a workgroup's share 4096; samples of just as many and one more, one behind the other."""
    rows, channels, groups = 1 << 22, 16, 4
    long = [8191, 8192, 8193, 8194, 16384, 16385, 9000, 8200, 100000, 12345]
    cuts = sizes((5000, 200), *((1, n) for n in long[:5]), (100, 37), *((1, n) for n in long[5:]), (4000, 301))
    cuts = cuts[:-1] + sizes((1, cuts[-1]), (1, rows - cuts[-1] - 10))[1:]
    assert len(cuts) - 1 >= 8192 and cuts == sorted(cuts)
    gen = torch.Generator().manual_seed(1)
    x, g = (torch.randint(-3, 4, (rows, channels), generator=gen, dtype=torch.int8) for _ in range(2))
    xd, gd = x.to(DEV).to(torch.bfloat16), g.to(DEV).to(torch.bfloat16)
    where, batch = torch.tensor(cuts, device=DEV), len(cuts) - 1
    mean, rstd = torch.zeros(batch, groups, device=DEV), torch.ones(batch, groups, device=DEV)
    got = scnn.group_norm_bwd(xd, gd, groups, None, None, mean, rstd, offsets=where)
    want = (x[:cuts[-1]] * g[:cuts[-1]]).sum(0, dtype=torch.int64), g[:cuts[-1]].sum(0, dtype=torch.int64)
    assert all(int(w.abs().max()) < 1 << 24 for w in want)
    assert torch.equal(got[1].cpu(), want[0].float().to(torch.bfloat16)) and torch.equal(got[2].cpu(), want[1].float().to(torch.bfloat16))
    out, m, r = scnn.group_norm_fwd(xd, groups, offsets=where, act="silu")
    dx = scnn.group_norm_bwd(xd, gd, groups, None, None, m, r, offsets=where, act="silu")[0]
    for b in (0, 4999, 5000, 5001, 5002, 5003, 5004, 5050, 5105, 5106, 5108, 5109, 9000, batch - 1):
        rows_b = slice(cuts[b], cuts[b + 1])
        for what, a, w in zip(("out", "mean", "rstd"), (out[rows_b], m[b:b + 1], r[b:b + 1]),
                              ref.group_norm_fwd(xd[rows_b], groups, None, None, [(0, cuts[b + 1] - cuts[b])], 1e-5, "silu", torch.bfloat16)):
            ref.assert_within(a, w, what)
        w = ref.group_norm_bwd(xd[rows_b], gd[rows_b], groups, None, None, m[b:b + 1], r[b:b + 1], [(0, cuts[b + 1] - cuts[b])], "silu", torch.bfloat16)
        ref.assert_within(dx[rows_b], w[0], "dx")


def test_a_nan_stays_in_its_sample_and_group():
    rows, channels, groups, offsets = CASES[3]
    d = make(7, rows, channels, torch.float32)
    where = torch.tensor(offsets, device=DEV)
    clean = scnn.group_norm_fwd(d["x"], groups, d["gamma"], d["beta"], offsets=where)
    for at in (5, 3000, 7099 + 6900, rows - 1):  # a short sample, a long one, the last row of the next, the last
        b = next(i for i in range(len(offsets) - 1) if offsets[i] <= at < offsets[i + 1])
        x = d["x"].clone()
        x[at, 12] = float("nan")
        out, mean, rstd = scnn.group_norm_fwd(x, groups, d["gamma"], d["beta"], offsets=where)
        hit = torch.zeros(rows, channels, dtype=torch.bool, device=DEV)
        hit[offsets[b]:offsets[b + 1], 10:15] = True
        assert bool(out[hit].isnan().all()) and torch.equal(out[~hit], clean[0][~hit])
        dx, dgamma, dbeta = scnn.group_norm_bwd(x, d["g"], groups, d["gamma"], d["beta"], mean, rstd, offsets=where)
        assert bool(dx[hit].isnan().all()) and bool(dx[~hit].isfinite().all()) and torch.equal(dgamma.isnan(), hit.any(0))


@pytest.mark.parametrize("k", (0, 3, 6, 9))
def test_a_workspace_of_the_size_asked_for(k):
    """Nothing is written beside it, and what it held before does not matter."""
    rows, channels, groups, offsets = CASES[k]
    d = make(3, rows, channels, torch.float32)
    where, batch = torch.tensor(offsets, device=DEV), len(offsets) - 1

    def both(rooms):
        y, m, r = scnn.group_norm_fwd(d["x"], groups, d["gamma"], d["beta"], offsets=where, act="silu", workspace=rooms[0])
        dx, dgamma, dbeta = scnn.group_norm_bwd(d["x"], d["g"], groups, d["gamma"], d["beta"], m, r, offsets=where, act="silu", workspace=rooms[1])
        return [y[offsets[0]:offsets[-1]], m, r, dx[offsets[0]:offsets[-1]], dgamma, dbeta]

    want = both((None, None))
    for fill in (0xA5, 0xFF):
        held, rooms = [], []
        for query in (scnn.group_norm_fwd_workspace, scnn.group_norm_bwd_workspace):
            need = query(torch.float32, rows, batch, channels, groups)
            held.append(torch.full((need + 1024,), fill, dtype=torch.uint8, device=DEV))
            rooms.append(held[-1][512:512 + need])
        assert all(torch.equal(a, b) for a, b in zip(both(rooms), want))
        for whole, room in zip(held, rooms):
            assert bool((whole[:512] == fill).all()) and bool((whole[512 + room.numel():] == fill).all())


def test_calls_on_two_streams_at_once():
    rows, channels, groups, offsets = CASES[4]
    d = make(4, rows, channels, torch.bfloat16)
    cuts = [offsets, one_long(rows, len(offsets) - 1)]
    where = [torch.tensor(c, device=DEV) for c in cuts]

    def calls(k, stream=None):
        y, m, r = scnn.group_norm_fwd(d["x"], groups, d["gamma"], offsets=where[k], act="gelu", stream=stream)
        dx, *rest = scnn.group_norm_bwd(d["x"], d["g"], groups, d["gamma"], None, m, r, offsets=where[k], act="gelu", stream=stream)
        return [y[:cuts[k][-1]], m, r, dx[:cuts[k][-1]], *rest]  # (rows behind the last sample are not written)

    want = [calls(k) for k in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = [calls(k, streams[k]) for k in range(2)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_numbers_that_do_not_ascend_end():
    """No defined result, but an end to the call."""
    rows, channels = 40000, 16
    d = make(5, rows, channels, torch.bfloat16)
    for bad in ([30000, 100, 40000, 0] * 16, [1 << 50, -(1 << 50), 7, 39000] * 16, list(range(rows, 0, -600))):
        t = torch.tensor(bad, device=DEV)
        out, mean, rstd = scnn.group_norm_fwd(d["x"], 4, d["gamma"], d["beta"], offsets=t)
        scnn.group_norm_bwd(d["x"], d["g"], 4, d["gamma"], d["beta"], mean, rstd, offsets=t)
    torch.cuda.synchronize()


def test_captured_and_replayed_with_other_sizes():
    """One graph for whatever the samples' sizes are: equal ones, one long one, none above the division."""
    rows, channels, groups, batch = 30000, 24, 6, 40
    d = make(31, rows, channels, torch.float32)
    offsets = torch.tensor([rows // batch * b for b in range(batch + 1)], device=DEV)
    outs = (torch.empty((rows, channels), device=DEV), torch.empty((batch, groups), device=DEV), torch.empty((batch, groups), device=DEV))
    grads = (torch.empty((rows, channels), device=DEV), torch.empty(channels, device=DEV), torch.empty(channels, device=DEV))

    def step():
        scnn.group_norm_fwd(d["x"], groups, d["gamma"], d["beta"], offsets=offsets, act="gelu", out=outs)
        scnn.group_norm_bwd(d["x"], d["g"], groups, d["gamma"], d["beta"], outs[1], outs[2], offsets=offsets, act="gelu", out=grads)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for cuts in (one_long(rows, batch), [rows // batch * b for b in range(batch + 1)], sizes((1, 12000), (1, 12000), (38, 100)), one_long(rows - 100, batch)):
        offsets.copy_(torch.tensor(cuts))
        for t in (*outs, *grads):
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*outs, *grads)]
        check(d, (rows, channels, groups, cuts), "gelu", d["gamma"], d["beta"], torch.float32)
        for t in (*outs, *grads):
            t.fill_(7.0)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*outs, *grads)))


@pytest.mark.parametrize("rows,channels,batch", [(131072, 16, 64), (262144, 64, 512)])
def test_a_long_sample_does_not_hold_the_call_up(rows, channels, batch):
    """One sample with all rows takes no more than ten times as long as equal ones (it took 35 and 140 times, left to one workgroup)."""
    d = make(9, rows, channels, torch.bfloat16)

    def took(cuts):
        offsets = torch.tensor(cuts, device=DEV)
        times = []
        for _ in range(9):
            first, last = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            first.record()
            for _ in range(10):
                y, m, r = scnn.group_norm_fwd(d["x"], 4, d["gamma"], d["beta"], offsets=offsets, act="silu")
                scnn.group_norm_bwd(d["x"], d["g"], 4, d["gamma"], d["beta"], m, r, offsets=offsets, act="silu")
            last.record()
            last.synchronize()
            times.append(first.elapsed_time(last))
        return statistics.median(times)

    assert took(sizes((batch // 2, 0), (1, rows), (batch - 1 - batch // 2, 0))) < 10 * took(sizes((batch, rows // batch)))
