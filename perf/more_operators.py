"""Timing cases of the layers that make a block on rows of values: group norm with its activation over the samples of a
sparse tensor, dropout whose mask is never stored, and linear layers in 8-bit integers for serving.

`run` computes each in its plain form, elementary operations in 32 bits (sums over a sample's rows and signs next to 0 in
64) rounded once at the end, or, with `own` set, by the library's calls; `exact` is the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "relu", "gelu", "silu")
# no drawn case is above these: the costliest listed product; three fifths of the bytes of the largest listed norm
MOST_FLOPS = 2.0 * 8192 * 4096 * 4096
MOST_BYTES = 200e6


def _norm(name, rows, batch, channels, groups, dtype, act, ragged=True, coords=False, back=False):
    return {"name": name, "kind": "group_norm_bwd" if back else "group_norm_fwd", "rows": rows, "batch": batch,
            "channels": channels, "groups": groups, "dtype": dtype, "act": act, "ragged": ragged, "coords": coords}


def _drop(name, rows, channels, dtype, p, residual=False, back=False):
    return {"name": name, "kind": "dropout_bwd" if back else "dropout_fwd", "rows": rows, "channels": channels,
            "dtype": dtype, "p": p, "residual": residual}


def _int8(name, rows, c_in, c_out, dtype, act, residual=False, given=False):
    return {"name": name, "kind": "linear_int8", "rows": rows, "c_in": c_in, "c_out": c_out, "dtype": dtype, "act": act,
            "residual": residual, "given": given}


def listed():
    return [
        # the sparse part's last maps (24 channels on 8^3 sites) of one sample: the smallest call of a served network
        _norm("norm_1x512x24", 512, 1, 24, 8, "fp32", "silu", ragged=False),
        # a batch of eight 32^3 samples of unequal sizes behind a sixteen-channel convolution, 16 bits
        _norm("norm_8_samples_23651x16", 23651, 8, 16, 4, "bf16", "gelu"),
        # rows of the benchmark layer's output, four samples, their bounds found in the coordinates on the way
        _norm("norm_643072x64", 643072, 4, 64, 8, "fp32", "relu", coords=True),
        # rows of the 128^3 network's input with an odd number of channels, backward: long sums over rows
        _norm("norm_bwd_209645x25", 209645, 2, 25, 5, "fp32", "relu", back=True),
        # dense maps, channels last: 64 samples of 8^3 sites, backward in 16 bits
        _norm("norm_bwd_64x512x256", 64 * 512, 64, 256, 32, "bf16", "silu", ragged=False, back=True),
        # hidden values of a fully connected layer on a training batch: latency
        _drop("drop_64x1024", 64, 1024, "fp32", 0.5),
        # rows of a wide block before its input is added, 16 bits
        _drop("drop_8192x4096", 8192, 4096, "bf16", 0.1, residual=True),
        # gradients on rows of a sparse tensor, an odd number of channels
        _drop("drop_bwd_643072x35", 643072, 35, "fp16", 0.2, back=True),
        # one row through a wide layer: weights read once, latency
        _int8("int8_1x4096_4096", 1, 4096, 4096, "bf16", "silu"),
        # first fully connected layer behind sparse_to_dense (24 channels on 8^3 sites) on a batch of 64
        _int8("int8_64x12288_1024", 64, 12288, 1024, "fp16", "relu"),
        # odd widths, rows that were brought to 8 bits for an earlier layer
        _int8("int8_3001x1001_1303", 3001, 1001, 1303, "fp32", "none", given=True),
        # a wide layer on a large batch, bound by the matrix cores
        _int8("int8_8192x4096_4096", 8192, 4096, 4096, "bf16", "gelu", residual=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("group_norm_fwd", "group_norm_fwd", "group_norm_bwd", "group_norm_bwd", "dropout_fwd", "dropout_bwd",
                       "linear_int8", "linear_int8", "linear_int8"))
    dtype = rng.choice(tuple(DTYPES))
    while True:
        if kind.startswith("group_norm"):
            channels = _log(rng, 1, 2048)
            if rng.random() < 0.5:  # layers are mostly a multiple of eight wide
                channels = -(-channels // 8) * 8
            groups = rng.choice([g for g in range(1, channels + 1) if channels % g == 0])
            batch, ragged = _log(rng, 1, 64), rng.random() < 0.7
            rows = _log(rng, 1, 700000)
            if not ragged:
                rows = -(-rows // batch) * batch
            case = _norm("", rows, batch, channels, groups, dtype, rng.choice(ACTS), ragged, ragged and rng.random() < 0.3,
                         kind == "group_norm_bwd")
        elif kind.startswith("dropout"):
            back = kind == "dropout_bwd"
            case = _drop("", _log(rng, 1, 700000), _log(rng, 1, 16384), dtype, round(rng.uniform(0.02, 0.9), 4),
                         not back and rng.random() < 0.5, back)
        else:
            size = (_log(rng, 1, 8192), _log(rng, 16, 16384), _log(rng, 10, 4096))
            if rng.random() < 0.5:
                size = (size[0], -(-size[1] // 8) * 8, -(-size[2] // 8) * 8)
            if 2.0 * math.prod(size) > MOST_FLOPS:
                continue
            case = _int8("", *size, dtype, rng.choice(ACTS), rng.random() < 0.5, rng.random() < 0.3)
        if work(case)["bytes"] <= MOST_BYTES:
            del case["name"]
            return case


def work(case):
    e = torch.empty(0, dtype=DTYPES[case["dtype"]]).element_size()
    r = case["rows"]
    if case["kind"] == "linear_int8":
        k, n = case["c_in"], case["c_out"]
        x = r * k + 4 * r if case["given"] else r * k * e
        return {"bytes": x + k * n + 4 * n + (n + (1 + case["residual"]) * r * n) * e, "flops": 2 * r * k * n}
    c = case["channels"]
    if case["kind"].startswith("dropout"):
        return {"bytes": (2 + case["residual"]) * r * c * e, "flops": 2 * r * c}
    stats = 8 * case["batch"] * (case["groups"] + 1) + (4 * r if case["coords"] else 0)
    if case["kind"] == "group_norm_fwd":
        return {"bytes": (2 * r * c + 2 * c) * e + stats, "flops": 8 * r * c}
    return {"bytes": (3 * r * c + 4 * c) * e + stats, "flops": 16 * r * c}


def _bounds(case, seed):
    """First rows of the samples: equal ones, or unequal ones of which some may be empty."""
    rows, batch = case["rows"], case["batch"]
    if not case["ragged"]:
        return [rows // batch * b for b in range(batch + 1)]
    rng = np.random.default_rng(seed)
    # (sizes of surfaces: alike within a factor of two or so; few rows leave samples without one)
    share = np.cumsum(rng.uniform(0.5, 1.5, batch))
    return [0] + [int(v) for v in np.round(share / share[-1] * rows)]


def _quantize(x):
    """Rows of values between -127 and 127: the values and what one step of each row stands for."""
    most = x.float().abs().amax(1, keepdim=True).clamp(min=2.0 ** -100)
    steps = torch.full_like(most, 127.0)  # (a number in its place would be divided by as a product with its inverse)
    return torch.round(x.float() * torch.div(steps, most)), torch.div(most, steps)


def _padded(q):
    """As int8, each row filled up with zeros to a multiple of 64."""
    out = torch.zeros(q.shape[0], -(-q.shape[1] // 64) * 64, dtype=torch.int8, device=q.device)
    out[:, :q.shape[1]] = q.to(torch.int8)
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(dt)

    state = {"case": case}
    rows = case["rows"]
    if case["kind"].startswith("dropout"):
        x = normal(rows, case["channels"])
        state |= {"x": x, "residual": normal(rows, case["channels"]) if case["residual"] else None, "seed": 1234567890123 + seed,
                  "offset": (1 << 40) + 3 * seed}
        return state
    if case["kind"] == "linear_int8":
        k, n = case["c_in"], case["c_out"]
        # (activations behind a ReLU: half of them 0)
        x = normal(rows, k).clamp_(min=0)
        q, scale = _quantize(normal(n, k, scale=math.sqrt(2.0 / k)))
        state |= {"w": _padded(q), "w_scale": scale[:, 0].contiguous(), "bias": normal(n, scale=0.1),
                  "residual": normal(rows, n) if case["residual"] else None, "x": x, "x_scale": None}
        if case["given"]:
            q, scale = _quantize(x)
            state |= {"x": _padded(q), "x_scale": scale[:, 0].contiguous()}
        return state
    c, batch, groups = case["channels"], case["batch"], case["groups"]
    bounds = _bounds(case, seed)
    offsets = torch.tensor(bounds, dtype=torch.int64, device="cuda")
    # (rows of activations: not centred)
    state |= {"x": normal(rows, c, scale=1.5, shift=0.5), "gamma": normal(c, scale=0.1, shift=1.0), "beta": normal(c, scale=0.1),
              "eps": 1e-5, "bounds": bounds, "offsets": offsets if case["ragged"] else None}
    if case["coords"]:
        site = torch.arange(rows, device="cuda", dtype=torch.int64)
        sample = torch.searchsorted(offsets[1:], site, right=True)
        at = site - offsets[sample]
        state["coords"] = torch.stack([sample, at >> 12, (at >> 6) & 63, at & 63], 1).to(torch.int32)
        state["offsets"] = None
    if case["kind"] == "group_norm_bwd":
        state["g"] = normal(rows, c, scale=0.1)
        mean = torch.zeros(batch, groups, dtype=torch.float64, device="cuda")
        rstd = torch.zeros_like(mean)
        for b in range(batch):
            if bounds[b + 1] > bounds[b]:
                v = state["x"][bounds[b]:bounds[b + 1]].double().view(-1, groups, c // groups)
                mean[b] = v.mean((0, 2))
                rstd[b] = ((v - mean[b, :, None]).square_().mean((0, 2)) + state["eps"]).rsqrt_()
        state |= {"mean": mean.float(), "rstd": rstd.float()}
    return state


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _dropped(n, case, seed, offset, device):
    """Which of n values are dropped: Philox 4x32 in ten rounds, eight values of 16 bits a counter."""
    low = 0xffffffff
    i = torch.arange(-(-n // 8), dtype=torch.int64, device=device)
    c = [i & low, i >> 32, torch.full_like(i, offset & low), torch.full_like(i, offset >> 32)]
    key = [seed & low, seed >> 32]
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57  # (64 bits, wrapped: the bits are those of the unsigned product)
        c = [((p1 >> 32) & low) ^ c[1] ^ key[0], p1 & low, ((p0 >> 32) & low) ^ c[3] ^ key[1], p0 & low]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    words = torch.stack([h for v in c for h in (v & 0xffff, v >> 16)], 1)
    return words.view(-1)[:n] < round(case["p"] * 65536)


def _run_plain(state):
    case = state["case"]
    dt = DTYPES[case["dtype"]]
    if case["kind"].startswith("dropout"):
        x = state["x"].float()
        drop = _dropped(x.numel(), case, state["seed"], state["offset"], x.device).view(x.shape)
        y = torch.where(drop, torch.zeros_like(x), x * (65536 / (65536 - round(case["p"] * 65536))))
        if state["residual"] is not None:
            y = y + state["residual"].float()
        return [y.to(dt)]
    if case["kind"] == "linear_int8":
        if case["given"]:
            q, scale = state["x"][:, :case["c_in"]].float(), state["x_scale"][:, None]
        else:
            q, scale = _quantize(state["x"])
        total = torch.zeros(case["rows"], case["c_out"], dtype=torch.int32, device=q.device)
        for k in range(0, case["c_in"], 1024):  # (whole numbers below 2^24: exact in 32 bits)
            to = min(case["c_in"], k + 1024)
            total += (q[:, k:to] @ state["w"][:, k:to].float().t()).to(torch.int32)
        y = _act(total.float() * scale * state["w_scale"] + state["bias"].float(), case["act"])
        if state["residual"] is not None:
            y = y + state["residual"].float()
        return [y.to(dt)]
    c, groups, bounds = case["channels"], case["groups"], state["bounds"]
    per = c // groups
    gamma, beta = state["gamma"].float(), state["beta"].float()
    if case["kind"] == "group_norm_fwd":
        out = torch.empty_like(state["x"])
        mean = torch.zeros(case["batch"], groups, device=out.device)
        rstd = torch.zeros_like(mean)
        for b in range(case["batch"]):
            if bounds[b + 1] == bounds[b]:
                continue
            x = state["x"][bounds[b]:bounds[b + 1]].double().view(-1, groups, per)
            m = x.mean((0, 2))
            d = x - m[:, None]
            r = 1 / torch.sqrt((d * d).mean((0, 2)) + state["eps"])
            z = (d.float() * r.float()[:, None]).view(-1, c) * gamma + beta
            out[bounds[b]:bounds[b + 1]] = _act(z, case["act"]).to(dt)
            mean[b], rstd[b] = m.float(), r.float()
        got = [out, mean, rstd]
        if case["coords"]:
            among = torch.arange(case["batch"] + 1, device=out.device, dtype=torch.int32)
            got.append((state["coords"][:, 0, None] < among).sum(0))
        return got
    dx = torch.empty_like(state["x"])
    dgamma = torch.zeros(c, dtype=torch.float64, device=dx.device)
    dbeta = torch.zeros_like(dgamma)
    for b in range(case["batch"]):
        if bounds[b + 1] == bounds[b]:
            continue
        part = slice(bounds[b], bounds[b + 1])
        # (the sign of z next to 0 decides relu's slope: 64 bits)
        xh = ((state["x"][part].double().view(-1, groups, per) - state["mean"][b][:, None].double())
              * state["rstd"][b][:, None].double()).view(-1, c)
        z = xh * gamma.double() + beta.double()
        dz = state["g"][part].float() * (_slope(z, "relu").float() if case["act"] == "relu" else _slope(z.float(), case["act"]))
        xh = xh.float()
        h = (dz * gamma).view(-1, groups, per)
        xg = xh.view(-1, groups, per)
        m_h, m_hx = h.double().mean((0, 2)).float(), (h * xg).double().mean((0, 2)).float()
        dx[part] = ((h - m_h[:, None] - xg * m_hx[:, None]) * state["rstd"][b][:, None]).view(-1, c).to(dt)
        dgamma += (dz * xh).double().sum(0)
        dbeta += dz.double().sum(0)
    return [dx, dgamma.to(dt), dbeta.to(dt)]


def _run_own(state):
    import paper_1801_10585_amd as scnn

    case = state["case"]
    if case["kind"] == "dropout_fwd":
        return [scnn.dropout_fwd(state["x"], case["p"], seed=state["seed"], offset=state["offset"], residual=state["residual"])]
    if case["kind"] == "dropout_bwd":
        return [scnn.dropout_bwd(state["x"], case["p"], seed=state["seed"], offset=state["offset"])]
    if case["kind"] == "linear_int8":
        return [scnn.linear_int8_fwd(state["x"], state["w"], state["w_scale"], state["bias"], x_scale=state["x_scale"],
                                     act=case["act"], residual=state["residual"], dtype=DTYPES[case["dtype"]])]
    offsets = state["offsets"]
    if case["coords"]:
        offsets = scnn.sample_offsets(state["coords"], case["batch"])
    if case["kind"] == "group_norm_fwd":
        got = scnn.group_norm_fwd(state["x"], case["groups"], state["gamma"], state["beta"], offsets=offsets,
                                  batch=case["batch"], eps=state["eps"], act=case["act"])
        return [*got, offsets] if case["coords"] else list(got)
    return list(scnn.group_norm_bwd(state["x"], state["g"], case["groups"], state["gamma"], state["beta"], state["mean"],
                                    state["rstd"], offsets=offsets, act=case["act"]))


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


def _kept(n, p, seed, offset):
    """The mask once more, on unsigned numbers: one array of counters [4, blocks]."""
    blocks = np.arange((n + 7) // 8, dtype=np.uint64)
    c = np.zeros((4, blocks.size), dtype=np.uint64)
    c[0], c[1], c[2], c[3] = blocks % 2 ** 32, blocks // 2 ** 32, offset % 2 ** 32, offset // 2 ** 32
    keys = np.uint64(seed % 2 ** 32), np.uint64(seed // 2 ** 32)
    s32, m32 = np.uint64(32), np.uint64(2 ** 32 - 1)
    for turn in range(10):
        k0 = (keys[0] + np.uint64(turn * 0x9E3779B9)) & m32
        k1 = (keys[1] + np.uint64(turn * 0xBB67AE85)) & m32
        first, second = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = np.stack([(second >> s32) ^ c[1] ^ k0, second & m32, (first >> s32) ^ c[3] ^ k1, first & m32])
    words = np.ascontiguousarray(c.T.astype(np.uint32)).view(np.uint16).reshape(-1)[:n]  # (low half of a word first)
    return torch.from_numpy(words >= int(round(p * 65536))).cuda()


def exact(case, seed):
    state = prepare(case, seed)
    wide = {k: v.double() for k, v in state.items() if torch.is_tensor(v) and v.is_floating_point()}
    if case["kind"].startswith("dropout"):
        x = wide["x"]
        keep = 1 - int(round(case["p"] * 65536)) / 65536
        y = torch.zeros_like(x)
        kept = _kept(x.numel(), case["p"], state["seed"], state["offset"]).view(x.shape)
        y[kept] = x[kept] / keep
        return [y if state["residual"] is None else y.add_(wide["residual"])]
    if case["kind"] == "linear_int8":
        k = case["c_in"]
        if case["given"]:
            q, step = state["x"][:, :k].double(), wide["x_scale"]
        else:
            # (the step and its inverse are held in 32 bits, and so is a value's quotient before it is rounded)
            most = torch.linalg.vector_norm(wide["x"], math.inf, dim=1).clamp_min(2.0 ** -100)
            step, inverse = (most / 127).float().double(), (127 / most).float().double()
            q = (wide["x"] * inverse[:, None]).float().double().round_()
        z = torch.mm(q, state["w"][:, :k].double().t().contiguous())
        z = torch.addcmul(wide["bias"], z, torch.outer(step, wide["w_scale"]))
        y = {"none": z, "relu": z * (z > 0), "gelu": z * torch.special.ndtr(z), "silu": z * torch.sigmoid(z)}[case["act"]]
        return [y if state["residual"] is None else y + wide["residual"]]
    c, groups, batch = case["channels"], case["groups"], case["batch"]
    per, bounds = c // groups, state["bounds"]
    acts = {"none": lambda z: z * 1, "relu": lambda z: z * (z > 0), "gelu": lambda z: z * torch.special.ndtr(z),
            "silu": lambda z: z * torch.sigmoid(z)}
    if case["kind"] == "group_norm_fwd":
        out, mean, rstd = torch.empty_like(wide["x"]), torch.zeros(batch, groups).double().cuda(), torch.zeros(batch, groups).double().cuda()
        for b in range(batch):
            lo, hi = bounds[b], bounds[b + 1]
            for j in range(groups if hi > lo else 0):
                cols = slice(j * per, (j + 1) * per)
                v = wide["x"][lo:hi, cols]
                var, m = torch.var_mean(v, correction=0)
                mean[b, j], rstd[b, j] = m, torch.rsqrt(var + state["eps"])
                out[lo:hi, cols] = acts[case["act"]](torch.addcmul(wide["beta"][cols], v - m, rstd[b, j] * wide["gamma"][cols]))
        return [out, mean, rstd] + ([torch.tensor(bounds, device="cuda")] if case["coords"] else [])
    dx = torch.empty_like(wide["x"])
    sums = torch.zeros(2, c, dtype=torch.float64, device="cuda")
    for b in range(batch):
        lo, hi = bounds[b], bounds[b + 1]
        if lo == hi:
            continue
        mean, rstd = (wide[k][b].repeat_interleave(per) for k in ("mean", "rstd"))
        xh = (wide["x"][lo:hi] - mean) * rstd
        z = torch.addcmul(wide["beta"], xh, wide["gamma"]).requires_grad_()
        dz, = torch.autograd.grad(acts[case["act"]](z), z, wide["g"][lo:hi])
        both = torch.stack([(dz * xh).sum(0), dz.sum(0)])
        sums += both
        # sums of a group's h and h xh are those of its columns times gamma
        of = (both * wide["gamma"]).view(2, groups, per).sum(2).repeat_interleave(per, 1) / ((hi - lo) * per)
        dx[lo:hi] = rstd * (dz * wide["gamma"] - of[1] - xh * of[0])
    return [dx, sums[0], sums[1]]
