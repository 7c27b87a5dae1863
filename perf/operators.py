"""Timing cases of the layers around the sparse part of a network, and of the step that closes a training pass.

Linear layers (matrix product with bias, activation and residual in one call) as they stand on the rows of a sparse
tensor and behind sparse_to_dense, layer norm of such rows, their gradients, and clipping of all gradients by their
global norm.  `run` computes each in its plain form, elementary operations in 32 bits rounded once at the end, or, with
`own` set, by the library's calls; `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "relu", "gelu", "silu")
# no drawn case is above these: the costliest listed product; four fifths of the bytes of the largest listed list of gradients
MOST_FLOPS = 4.0 * 4096 * 4096 * 4096
MOST_BYTES = 400e6
# layers (taps, channels in, channels out) of the nine-layer network of the paper's appendix
NET_LAYERS = ((27, 1, 8), (27, 8, 8), (27, 8, 8), (27, 8, 16), (27, 16, 16), (27, 16, 16), (27, 16, 24), (27, 24, 24),
              (27, 24, 24))


def _linear(name, rows, c_in, c_out, dtype, act, residual=False, keep=False, back=False):
    return {"name": name, "kind": "linear_bwd" if back else "linear_fwd", "rows": rows, "c_in": c_in, "c_out": c_out,
            "dtype": dtype, "act": act, "residual": residual, "keep": keep}


def _norm(name, rows, channels, dtype, back=False):
    return {"name": name, "kind": "layer_norm_bwd" if back else "layer_norm_fwd", "rows": rows, "channels": channels,
            "dtype": dtype}


def _clip(name, dtype, net, tensors, largest, max_norm):
    return {"name": name, "kind": "clip", "dtype": dtype, "net": net, "tensors": tensors, "largest": largest,
            "max_norm": max_norm}


def listed():
    return [
        # class scores of one sample: the smallest call of a served network, launches and latency
        _linear("scores_1x1024_40", 1, 1024, 40, "fp32", "none"),
        # first fully connected layer behind sparse_to_dense (24 channels on 8^3 sites) on a training batch: weights
        # read once for 64 rows
        _linear("head_64x12288_1024", 64, 12288, 1024, "fp32", "relu", keep=True),
        # a linear layer on the rows of the benchmark's sparse tensor, its input added: many rows, few channels
        _linear("sites_202470x32_64", 202470, 32, 64, "fp32", "relu", residual=True),
        # a wide layer on a large batch in 16 bits, bound by the matrix cores
        _linear("wide_8192x4096_4096", 8192, 4096, 4096, "bf16", "gelu", residual=True, keep=True),
        # gradients of a narrow layer of odd widths on rows of a sparse tensor: a long sum over rows, 19 classes a site
        _linear("sites_bwd_52417x35_19", 52417, 35, 19, "fp16", "silu", back=True),
        # gradients of the wide layer: two products
        _linear("wide_bwd_4096x4096_4096", 4096, 4096, 4096, "bf16", "gelu", back=True),
        # one row: the smallest normalisation of a served network
        _norm("norm_1x1024", 1, 1024, "fp16"),
        # rows of the benchmark layer's output: many short rows
        _norm("norm_643072x64", 643072, 64, "fp32"),
        # rows of the 128^3 network's input with an odd number of channels, backward: a long sum over rows
        _norm("norm_bwd_209645x25", 209645, 25, "fp32", back=True),
        # wide rows in 16 bits, backward
        _norm("norm_bwd_8192x4096", 8192, 4096, "bf16", back=True),
        # all gradients of the nine-layer network: 18 small tensors, latency
        _clip("clip_nine_layers", "fp32", True, 0, 0, 0.5),
        # gradients of a model of 60 tensors, 127 M entries in all
        _clip("clip_60_tensors", "bf16", False, 60, 12000000, 1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("linear_fwd", "linear_fwd", "linear_bwd", "linear_bwd", "layer_norm_fwd", "layer_norm_bwd", "clip"))
    dtype = rng.choice(tuple(DTYPES))
    while True:
        if kind == "clip":
            net = rng.random() < 0.2
            case = _clip("", dtype, net, 0 if net else _log(rng, 1, 60), 0 if net else _log(rng, 100, 12000000),
                         round(rng.uniform(0.1, 10.0), 3))
        elif kind.startswith("linear"):
            place = rng.choice(("head", "sites", "wide"))
            if place == "head":
                size = (_log(rng, 1, 256), _log(rng, 64, 16384), _log(rng, 10, 4096))
            elif place == "sites":
                size = (_log(rng, 500, 300000), _log(rng, 1, 128), _log(rng, 1, 128))
            else:
                size = (_log(rng, 256, 8192), _log(rng, 128, 4096), _log(rng, 128, 4096))
            if rng.random() < 0.5:  # layers are mostly a multiple of eight wide
                size = (size[0], -(-size[1] // 8) * 8, -(-size[2] // 8) * 8)
            act = rng.choice(ACTS)
            back = kind == "linear_bwd"
            case = _linear("", *size, dtype, act, not back and rng.random() < 0.5, not back and rng.random() < 0.5, back)
            # (products of 32 bits cost several times those of 16)
            if 2.0 * math.prod(size) * (2 if back else 1) > MOST_FLOPS / (4 if dtype == "fp32" else 1):
                continue
        else:
            channels = _log(rng, 1, 16384)
            rows = _log(rng, 1, max(1, min(700000, 40000000 // channels)))
            case = _norm("", rows, channels, dtype, kind.endswith("bwd"))
        if work(case)["bytes"] <= MOST_BYTES:
            del case["name"]
            return case


def _clip_shapes(case):
    if case["net"]:
        return [(t, i, o) for t, i, o in NET_LAYERS] + [(o,) for _, _, o in NET_LAYERS]
    shapes = []
    for k in range(case["tensors"]):
        # matrices of a model between vectors of its biases and norms, in sizes that fall with the depth
        n = max(1, case["largest"] >> (k % 8)) if k % 2 == 0 else max(1, int(math.sqrt(case["largest"])) - k % 3)
        shapes.append((n,))
    return shapes


def _size(case):
    return torch.empty(0, dtype=DTYPES[case["dtype"]]).element_size()


def work(case):
    e = _size(case)
    if case["kind"] == "clip":
        n = sum(math.prod(s) for s in _clip_shapes(case))
        return {"bytes": 2 * n * e, "flops": 3 * n}
    r = case["rows"]
    if case["kind"].startswith("layer_norm"):
        c = case["channels"]
        if case["kind"] == "layer_norm_fwd":
            return {"bytes": (2 * r * c + 2 * c) * e + 8 * r, "flops": 8 * r * c}
        return {"bytes": (3 * r * c + 3 * c) * e + 8 * r, "flops": 14 * r * c}
    k, n = case["c_in"], case["c_out"]
    if case["kind"] == "linear_fwd":
        outs = 1 + case["keep"] + case["residual"]
        return {"bytes": (r * k + k * n + n + outs * r * n) * e, "flops": 2 * r * k * n}
    reads = r * k + k * n + (1 + (case["act"] != "none")) * r * n
    return {"bytes": (reads + r * k + k * n + n) * e, "flops": 4 * r * k * n}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(dt)

    state = {"case": case}
    if case["kind"] == "clip":
        state["grads"] = [normal(*s, scale=0.02) for s in _clip_shapes(case)]
        state["outs"] = [torch.empty_like(g) for g in state["grads"]]
        return state
    rows = case["rows"]
    if case["kind"].startswith("layer_norm"):
        c = case["channels"]
        # (rows of activations: not centred, of different sizes)
        x = normal(rows, c, scale=1.5, shift=0.5)
        state |= {"x": x, "gamma": normal(c, scale=0.1, shift=1.0), "beta": normal(c, scale=0.1), "eps": 1e-5}
        if case["kind"] == "layer_norm_bwd":
            state["g"] = normal(rows, c, scale=0.1)
            v = x.double()
            mean = v.mean(1)
            var = (v - mean[:, None]).square_().mean(1)
            state |= {"mean": mean.float(), "rstd": (var + state["eps"]).rsqrt_().float()}
        return state
    k, n = case["c_in"], case["c_out"]
    # (activations behind a ReLU: half of them 0)
    state |= {"x": normal(rows, k).clamp_(min=0), "w": normal(k, n, scale=math.sqrt(2.0 / k)), "bias": normal(n, scale=0.1)}
    state["residual"] = normal(rows, n) if case["residual"] else None
    if case["kind"] == "linear_bwd":
        state["g"] = normal(rows, n, scale=0.1)
        state["pre"] = (state["x"].float() @ state["w"].float() + state["bias"].float()).to(dt)
    return state


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_gradient(g, z, act):
    if act == "relu":
        return torch.where(z <= 0, torch.zeros_like(g), g)
    if act == "gelu":
        return g * (0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi))
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return g * (s * (1 + z * (1 - s)))
    return g


def _run_plain(state):
    case = state["case"]
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "clip":
        # (squares of long tensors, some past the largest number of 32 bits: summed in 64)
        norm = torch.stack([g.double().square().sum() for g in state["grads"]]).sum().sqrt()
        scale = torch.clamp(case["max_norm"] / (norm + 1e-6), max=1.0)
        by = scale.float()
        return [norm, scale, [(g.float() * by).to(dt) for g in state["grads"]]]
    x = state["x"].float()
    if case["kind"] == "linear_fwd":
        z = x @ state["w"].float() + state["bias"].float()
        y = _act(z, case["act"])
        if case["residual"]:
            y = y + state["residual"].float()
        return [y.to(dt), z.to(dt)] if case["keep"] else [y.to(dt)]
    if case["kind"] == "linear_bwd":
        dz = _act_gradient(state["g"].float(), state["pre"].float(), case["act"])
        return [(dz @ state["w"].float().t()).to(dt), (x.t() @ dz).to(dt), dz.sum(0).to(dt)]
    if case["kind"] == "layer_norm_fwd":
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + state["eps"])
        y = d * rstd * state["gamma"].float() + state["beta"].float()
        return [y.to(dt), mean[:, 0], rstd[:, 0]]
    g, rstd = state["g"].float(), state["rstd"][:, None]
    xh = (x - state["mean"][:, None]) * rstd
    h = g * state["gamma"].float()
    dx = rstd * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    return [dx.to(dt), (g * xh).sum(0).to(dt), g.sum(0).to(dt)]


def _run_own(state):
    import paper_1801_10585_amd as scnn

    case = state["case"]
    if case["kind"] == "clip":
        result = scnn.clip_grad_norm(state["grads"], case["max_norm"], outs=state["outs"])
        return [result[0], result[1], state["outs"]]
    if case["kind"] == "linear_fwd":
        got = scnn.linear_fwd(state["x"], state["w"], state["bias"], act=case["act"], residual=state["residual"],
                              keep_pre=case["keep"])
        return list(got) if case["keep"] else [got]
    if case["kind"] == "linear_bwd":
        return list(scnn.linear_bwd(state["x"], state["w"], state["g"], act=case["act"],
                                    pre=None if case["act"] == "none" else state["pre"]))
    if case["kind"] == "layer_norm_fwd":
        return list(scnn.layer_norm_fwd(state["x"], state["gamma"], state["beta"], eps=state["eps"]))
    return list(scnn.layer_norm_bwd(state["x"], state["g"], state["gamma"], state["mean"], state["rstd"]))


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


def exact(case, seed):
    state = prepare(case, seed)
    wide = {k: v.double() for k, v in state.items() if torch.is_tensor(v)}
    if case["kind"] == "clip":
        grads = [g.double() for g in state["grads"]]
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g)) ** 2 for g in grads))
        scale = min(1.0, case["max_norm"] / (norm + 1e-6))
        one = torch.ones((), dtype=torch.float64, device="cuda")
        return [one * norm, one * scale, [g.mul_(scale) for g in grads]]
    if case["kind"] == "linear_fwd":
        z = torch.addmm(wide["bias"], wide["x"], wide["w"])
        y = {"none": z, "relu": z * (z > 0), "gelu": z * torch.special.ndtr(z), "silu": z * torch.sigmoid(z)}[case["act"]]
        if case["residual"]:
            y = y + wide["residual"]
        return [y, z] if case["keep"] else [y]
    if case["kind"] == "linear_bwd":
        z = wide["pre"].requires_grad_()
        y = {"none": z * 1, "relu": z * (z > 0), "gelu": z * torch.special.ndtr(z), "silu": z * torch.sigmoid(z)}[case["act"]]
        dz, = torch.autograd.grad(y, z, wide["g"])
        return [torch.mm(dz, wide["w"].t().contiguous()), torch.mm(wide["x"].t().contiguous(), dz), dz.sum(0)]
    x = wide["x"]
    if case["kind"] == "layer_norm_fwd":
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = torch.rsqrt(var + state["eps"])
        return [(x - mean[:, None]) * (rstd[:, None] * wide["gamma"]) + wide["beta"], mean, rstd]
    mean, rstd, g = wide["mean"][:, None], wide["rstd"][:, None], wide["g"]
    # the Jacobian of one row applied to h: rstd (I - 1 1^T / C - xh xh^T / C) h
    xh = (x - mean) * rstd
    h = g * wide["gamma"]
    c = x.shape[1]
    dx = (h - h.sum(1, keepdim=True) / c - xh * (torch.linalg.vecdot(xh, h, dim=1)[:, None] / c)) * rstd
    return [dx, (xh * g).sum(0), g.sum(0)]
