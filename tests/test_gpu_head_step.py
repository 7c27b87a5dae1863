"""The row layers, their gradients and the clipping together, as a training step uses them: a convolution's output rows
through layer norm and a per-site linear layer with its input added, sparse_to_dense, two fully connected layers with layer
norm between them, the gradients all the way back to the rows, and one clipping of all of them."""
import pytest
import torch

import paper_1801_10585_amd as scnn
from workloads import make_config
from . import rows_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EXT, BATCH, CH, HIDDEN, CLASSES = (8, 8, 8), 4, 24, 72, 10


def parameters(seed):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, s=1.0, m=0.0):
        return (torch.randn(*shape, generator=g) * s + m).to(DEV)

    flat = CH * EXT[0] * EXT[1] * EXT[2]
    return {"gamma0": normal(CH, s=0.1, m=1.0), "beta0": normal(CH, s=0.1), "w0": normal(CH, CH, s=CH ** -0.5),
            "b0": normal(CH, s=0.1), "w1": normal(flat, HIDDEN, s=0.05), "b1": normal(HIDDEN, s=0.1),
            "gamma1": normal(HIDDEN, s=0.1, m=1.0), "beta1": normal(HIDDEN, s=0.1), "w2": normal(HIDDEN, CLASSES, s=0.1),
            "b2": normal(CLASSES, s=0.1)}


def conv_rows(seed):
    wl = make_config(2, r=8, batch=BATCH, seed=seed)
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(27, wl.feats.shape[1], CH, generator=g).to(DEV) * 0.1
    c, f = torch.from_numpy(wl.coords).to(DEV), torch.from_numpy(wl.feats).to(DEV)
    return scnn.sparse_conv_fwd(EXT, BATCH, c, f, (3, 3, 3), w, rho_up=0.5, relu=True,
                                out_capacity=BATCH * 512, sync=False)


def step(p, coords, rows, rows_dev, labels, hot):
    """Logits and gradients by the library's calls; `rows` at their capacity, the count on the device."""
    n0, m0, r0 = scnn.layer_norm_fwd(rows, p["gamma0"], p["beta0"], rows_dev=rows_dev)
    s0, z0 = scnn.linear_fwd(n0, p["w0"], p["b0"], act="silu", residual=rows, keep_pre=True, rows_dev=rows_dev)
    dense = scnn.sparse_to_dense(EXT, BATCH, coords, s0, rows_dev=rows_dev)
    flat = dense.view(BATCH, -1)
    h1, z1 = scnn.linear_fwd(flat, p["w1"], p["b1"], act="gelu", keep_pre=True)
    n1, m1, r1 = scnn.layer_norm_fwd(h1, p["gamma1"], p["beta1"])
    logits = scnn.linear_fwd(n1, p["w2"], p["b2"])
    d = (torch.softmax(logits, 1) - hot) / BATCH  # of the mean cross-entropy
    g = {}
    dn1, g["w2"], g["b2"] = scnn.linear_bwd(n1, p["w2"], d)
    dh1, g["gamma1"], g["beta1"] = scnn.layer_norm_bwd(h1, dn1, p["gamma1"], m1, r1)
    dflat, g["w1"], g["b1"] = scnn.linear_bwd(flat, p["w1"], dh1, act="gelu", pre=z1)
    # the gradient of sparse_to_dense: each row takes its site's channels
    at = coords.long()
    ds0 = dflat.view(BATCH, CH, *EXT)[at[:, 0].clamp(0, BATCH - 1), :, at[:, 1].clamp(0, 7), at[:, 2].clamp(0, 7),
                                      at[:, 3].clamp(0, 7)].contiguous()
    dn0, g["w0"], g["b0"] = scnn.linear_bwd(n0, p["w0"], ds0, act="silu", pre=z0, rows_dev=rows_dev)
    drows, g["gamma0"], g["beta0"] = scnn.layer_norm_bwd(rows, dn0, p["gamma0"], m0, r0, rows_dev=rows_dev)
    return logits, g, drows, ds0


def reference(p, coords, rows, labels):
    """The same by automatic differentiation in 64 bits on the CPU."""
    q = {k: v.double().cpu().requires_grad_() for k, v in p.items()}
    x = rows.double().cpu().requires_grad_()
    at = coords.cpu().long()

    def norm(v, gamma, beta):
        m = v.mean(1, keepdim=True)
        return (v - m) / torch.sqrt(((v - m) ** 2).mean(1, keepdim=True) + 1e-5) * gamma + beta

    s0 = ref.act(norm(x, q["gamma0"], q["beta0"]) @ q["w0"] + q["b0"], "silu") + x
    dense = torch.zeros(BATCH, CH, *EXT, dtype=torch.float64)
    dense = dense.permute(0, 2, 3, 4, 1).index_put((at[:, 0], at[:, 1], at[:, 2], at[:, 3]), s0).permute(0, 4, 1, 2, 3)
    h1 = ref.act(dense.reshape(BATCH, -1) @ q["w1"] + q["b1"], "gelu")
    logits = norm(h1, q["gamma1"], q["beta1"]) @ q["w2"] + q["b2"]
    loss = -torch.log_softmax(logits, 1)[torch.arange(BATCH), labels.cpu()].mean()
    loss.backward()
    return logits.detach(), {k: v.grad for k, v in q.items()}, x.grad


def near(got, want, rel, what):
    """Of the tensor's own size: the sums behind an element are far shorter than 2^13 terms, each of a few U32."""
    got = got.double().cpu()
    assert float((got - want).norm()) <= rel * float(want.norm()), what


def labels_for(seed):
    labels = torch.randint(0, CLASSES, (BATCH,), generator=torch.Generator().manual_seed(seed)).to(DEV)
    return labels, torch.nn.functional.one_hot(labels, CLASSES).float()


# a chain of five layers of sums of up to 12288 products: some hundred roundings of 2^-24 on each, errors of different layers
# add up; layer norms divide by their rows' spread, which here is no less than a tenth of their size
REL = 100 * 5 * 10 * ref.U32


def test_a_training_step():
    p = parameters(1)
    coords, rows, nnz = conv_rows(3)
    n = int(nnz[0])
    assert 100 < n < rows.shape[0]
    rows[n:] = float("nan")
    coords[n:] = -1
    labels, hot = labels_for(5)
    logits, g, drows, ds0 = step(p, coords, rows, nnz[:1], labels, hot)
    want_logits, want, want_rows = reference(p, coords[:n], rows[:n], labels)
    near(logits, want_logits, REL, "logits")
    for k in p:
        near(g[k], want[k], REL, k)
    near(drows[:n] + ds0[:n], want_rows, REL, "rows")  # through the norm and past it
    # one clipping over all of them
    names = sorted(g)
    kept = {k: g[k].clone() for k in names}
    result = scnn.clip_grad_norm([g[k] for k in names], 0.1).cpu()
    norm = float(sum(kept[k].double().square().sum() for k in names).sqrt())
    assert float(result[0]) == pytest.approx(norm, rel=1e-12) and norm > 0.1
    assert float(result[0]) == pytest.approx(float(sum(w.square().sum() for w in want.values()).sqrt()), rel=REL)
    for k in names:
        assert torch.allclose(g[k], kept[k] * (0.1 / (norm + 1e-6)), rtol=4 * ref.U32, atol=0)
    assert float(scnn.grad_norm([g[k] for k in names])) == pytest.approx(0.1, rel=1e-5)


def test_the_step_captured_and_replayed():
    """One graph over everything that follows the convolution; every replay on other rows and another count."""
    p = parameters(2)
    coords, rows, nnz = conv_rows(7)
    labels, hot = labels_for(8)
    count = nnz[:1].clone()

    def both():
        logits, g, drows, _ = step(p, coords, rows, count, labels, hot)
        result = scnn.clip_grad_norm([g[k] for k in sorted(g)], 0.5)
        return [logits, drows, result] + [g[k] for k in sorted(g)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for seed in (11, 12, 13, 14):
        c, f, m = conv_rows(seed)
        coords.copy_(c)
        rows.copy_(f)
        count.copy_(m[:1])
        n = int(m[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        eager = both()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, eager)):
            if i == 1:
                a, b = a[:n], b[:n]
            assert torch.equal(a, b), (seed, i)
