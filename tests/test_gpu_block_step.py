"""Group norm, linear layers and dropout together as a block on a convolution's output rows: a training step with all gradients
and their clipping, eager and captured, and the same block served with 8-bit products."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from workloads import make_config
from . import block_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EXT, BATCH, CH, WIDE, GROUPS, P = (8, 8, 8), 4, 24, 40, 6, 0.3


def parameters(seed):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, s=1.0, m=0.0):
        return (torch.randn(*shape, generator=g) * s + m).to(DEV)

    return {"gamma": normal(CH, s=0.1, m=1.0), "beta": normal(CH, s=0.1), "w0": normal(CH, WIDE, s=CH ** -0.5), "b0": normal(WIDE, s=0.1),
            "w1": normal(WIDE, CH, s=WIDE ** -0.5), "b1": normal(CH, s=0.1)}


def conv_rows(seed):
    wl = make_config(2, r=8, batch=BATCH, seed=seed)
    w = torch.randn(27, wl.feats.shape[1], CH, generator=torch.Generator().manual_seed(seed)).to(DEV) * 0.1
    c, f = torch.from_numpy(wl.coords).to(DEV), torch.from_numpy(wl.feats).to(DEV)
    return scnn.sparse_conv_fwd(EXT, BATCH, c, f, (3, 3, 3), w, rho_up=0.5, relu=True, out_capacity=BATCH * 512, sync=False)


def step(p, coords, rows, count, up, rng):
    """rows + dropout(linear(linear(group norm))), and gradients from `up`; `rows` at their capacity, the count on the device."""
    offsets = scnn.sample_offsets(coords, BATCH, rows_dev=count)
    n, mean, rstd = scnn.group_norm_fwd(rows, GROUPS, p["gamma"], p["beta"], offsets=offsets, act="silu")
    h, z = scnn.linear_fwd(n, p["w0"], p["b0"], act="gelu", keep_pre=True, rows_dev=count)
    y = scnn.linear_fwd(h, p["w1"], p["b1"], rows_dev=count)
    out = scnn.dropout_fwd(y, P, rng=rng, residual=rows, rows_dev=count)
    g = {}
    dy = scnn.dropout_bwd(up, P, rng=rng, rows_dev=count)
    dh, g["w1"], g["b1"] = scnn.linear_bwd(h, p["w1"], dy, rows_dev=count)
    dn, g["w0"], g["b0"] = scnn.linear_bwd(n, p["w0"], dh, act="gelu", pre=z, rows_dev=count)
    drows, g["gamma"], g["beta"] = scnn.group_norm_bwd(rows, dn, GROUPS, p["gamma"], p["beta"], mean, rstd, offsets=offsets, act="silu")
    return out, g, drows


def reference(p, sample, rows, up, kept):
    q = {k: v.double().cpu().requires_grad_() for k, v in p.items()}
    x = rows.double().cpu().requires_grad_()
    parts = []
    for b in range(BATCH):
        v = x[sample == b].view(-1, GROUPS, CH // GROUPS)
        m = v.mean((0, 2), keepdim=True)
        parts.append(((v - m) / torch.sqrt(((v - m) ** 2).mean((0, 2), keepdim=True) + 1e-5)).view(-1, CH))
    n = ref.act(torch.cat(parts) * q["gamma"] + q["beta"], "silu")
    y = ref.act(n @ q["w0"] + q["b0"], "gelu") @ q["w1"] + q["b1"]
    scale = 65536 / (65536 - round(P * 65536))
    out = torch.where(kept, y * scale, torch.zeros(()).double()) + x
    (out * up.double().cpu()).sum().backward()
    return out.detach(), {k: v.grad for k, v in q.items()}, x.grad, n.detach()


def near(got, want, rel, what):
    got = got.double().cpu()
    assert float((got - want).norm()) <= rel * float(want.norm()), what


# a chain of four layers of sums of up to 2048 rows: some hundred roundings of 2^-24 on each, errors of different layers add up;
# norms divide by their samples' spread, which here is no less than a tenth of their size
REL = 100 * 4 * 10 * ref.U32


def test_a_training_step_and_the_served_block():
    p = parameters(1)
    coords, rows, nnz = conv_rows(3)
    n = int(nnz[0])
    assert 100 < n < rows.shape[0]
    rows[n:] = float("nan")
    up = torch.randn(rows.shape, generator=torch.Generator().manual_seed(2)).to(DEV)
    rng = torch.tensor([11, 5], device=DEV)
    kept = (ref.words(0, n * CH, 11, 5) >= round(P * 65536)).view(n, CH)
    out, g, drows = step(p, coords, rows, nnz[:1], up, rng)
    sample = coords[:n, 0].cpu()
    want, want_g, want_rows, want_n = reference(p, sample, rows[:n], up[:n], kept)
    near(out[:n], want, REL, "out")
    near(drows[:n] + up[:n], want_rows, REL, "rows")
    for k in p:
        near(g[k], want_g[k], REL, k)
    kept_g = {k: v.clone() for k, v in g.items()}
    norm = float(sum(w.square().sum() for w in want_g.values()).sqrt())
    result = scnn.clip_grad_norm([g[k] for k in sorted(g)], norm / 10).cpu()
    assert float(result[0]) == pytest.approx(norm, rel=REL)
    for k in p:
        assert torch.allclose(g[k], kept_g[k] * 0.1, rtol=REL, atol=0)
    # served: no dropout, both products in 8 bits
    q0, q1 = scnn.quantize_weight(p["w0"]), scnn.quantize_weight(p["w1"])
    offsets = scnn.sample_offsets(coords, BATCH, rows_dev=nnz[:1])
    norms = scnn.group_norm_fwd(rows, GROUPS, p["gamma"], p["beta"], offsets=offsets, act="silu")[0]
    h = scnn.linear_int8_fwd(norms, *q0, p["b0"], act="gelu", rows_dev=nnz[:1])
    served = scnn.linear_int8_fwd(h, *q1, p["b1"], residual=rows, rows_dev=nnz[:1])[:n]
    full = ref.act(want_n @ p["w0"].double().cpu() + p["b0"].double().cpu(), "gelu") @ p["w1"].double().cpu() + p["b1"].double().cpu()
    # a row's values are off by up to half a step of its largest, 1/254; two products of two such operands each, errors
    # spread evenly over a step: 4 x 1/254/sqrt(3) of the largest, about three times the mean magnitude: a tenth at the most
    near(served.double().cpu() - rows[:n].double().cpu(), full, 0.1, "served")
    # and exactly what the 8-bit operands give, layer by layer
    xq, xs = scnn.quantize_rows(norms[:n])
    ref.assert_within(h[:n], ref.linear_int8(xq, xs, *q0, p["b0"], "gelu", None, torch.float32))
    xq, xs = scnn.quantize_rows(h[:n])
    ref.assert_within(served, ref.linear_int8(xq, xs, *q1, p["b1"], "none", rows[:n], torch.float32))


def test_the_step_captured_and_replayed():
    """One graph over everything that follows the convolution; every replay on other rows, another count and another mask."""
    p = parameters(2)
    coords, rows, nnz = conv_rows(7)
    up = torch.randn(rows.shape, generator=torch.Generator().manual_seed(4)).to(DEV)
    count, rng = nnz[:1].clone(), torch.tensor([3, 0], device=DEV)

    def all_of_it():
        out, g, drows = step(p, coords, rows, count, up, rng)
        result = scnn.clip_grad_norm([g[k] for k in sorted(g)], 0.5)
        return [out, drows, result] + [g[k] for k in sorted(g)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_of_it()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = all_of_it()
    for k, seed in enumerate((11, 12, 13, 14)):
        c, f, m = conv_rows(seed)
        coords.copy_(c)
        rows.copy_(f)
        count.copy_(m[:1])
        rng.copy_(torch.tensor([3, k]))
        n = int(m[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        eager = all_of_it()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, eager)):
            if i < 2:
                a, b = a[:n], b[:n]
            assert torch.equal(a, b), (seed, i)
