"""Performance cases of the digital operators beside the crossbar layers: group norm with an activation, low-rank adapters, and the
global gradient norm with clipping and the clipped step.

Every case runs in its plain form (elementary torch operations) or, with `own` set, through the package's calls.  Sizes are those of
the benchmarked networks' layers (ResNet-20 and ResNet-50 activations, classifiers and fully connected layers of the perceptron, of
ResNet-50 and of VGG-16), with odd ones between them.
"""
import math
import random

import torch

own = False

ACTS = ("none", "relu", "silu")
EPS = 1e-5
LR, MAX_NORM = 0.01, 1.0


# ---- the cases -----------------------------------------------------------------------------------
def _gn(direction, batch, h, w, channels, groups, act, skip):
    return dict(op="gn_" + direction, batch=batch, h=h, w=w, channels=channels, groups=groups, act=act, skip=skip)


def _adapter(direction, rows, K, N, rank, adapters, requests, shuffled, bf16, plan):
    return dict(op="adapter_" + direction, rows=rows, K=K, N=N, rank=rank, adapters=adapters, requests=requests, shuffled=shuffled,
                bf16=bf16, plan=plan)


def _grads(kind, tensors, smallest, largest, layout):
    return dict(op="grads_" + kind, tensors=tensors, smallest=smallest, largest=largest, layout=layout)


def listed():
    return [
        # last stage of a ResNet-20, one image: the smallest call of a network that answers single requests
        dict(name="gn_fwd_one_image", **_gn("fwd", 1, 8, 8, 64, 16, "relu", False)),
        # ragged sizes and a residual branch under the smooth activation
        dict(name="gn_fwd_ragged_silu", **_gn("fwd", 13, 15, 17, 90, 9, "silu", True)),
        # the widest activations of a ResNet-50 at the benchmark's batch, with the residual branch
        dict(name="gn_fwd_resnet50_stage1", **_gn("fwd", 64, 56, 56, 256, 32, "relu", True)),
        # first stage of a ResNet-20 at its batch, backward
        dict(name="gn_bwd_resnet20", **_gn("bwd", 128, 32, 32, 16, 4, "relu", False)),
        # second stage of a ResNet-50, backward
        dict(name="gn_bwd_resnet50_stage2", **_gn("bwd", 64, 28, 28, 512, 32, "relu", False)),
        # one request at the ResNet-50 classifier: two short products, bound by their latency
        dict(name="adapter_fwd_one_row", **_adapter("fwd", 1, 2048, 1000, 8, 4, 1, False, False, False)),
        # 128 requests of one row each at a VGG-16 layer, in no order, compact adapters; the batch is a new one, so its plan counts too
        dict(name="adapter_fwd_128_requests", **_adapter("fwd", 128, 4096, 4096, 16, 64, 128, True, True, True)),
        # long requests, a few adapters: the rate of memory
        dict(name="adapter_fwd_long_requests", **_adapter("fwd", 4096, 4096, 4096, 32, 8, 20, False, False, False)),
        # training of a few adapters beside the first fully connected layer of a VGG-16, odd rank
        dict(name="adapter_bwd_vgg16_fc1", **_adapter("bwd", 128, 25088, 4096, 24, 3, 9, False, False, False)),
        # training of adapters with many rows
        dict(name="adapter_bwd_many_rows", **_adapter("bwd", 2048, 4096, 4096, 16, 4, 16, True, False, False)),
        # gamma and beta of a small network: many short tensors, bound by launches
        dict(name="grads_norm_short_tensors", **_grads("norm", 38, 16, 1000, 1)),
        # adapters and normalisations of a large network, one step of all of them
        dict(name="grads_step_large_network", **_grads("step", 54, 64, 6000000, 2)),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("gn_fwd", "gn_bwd", "adapter_fwd", "adapter_bwd", "grads"))
    while True:
        if kind.startswith("gn"):
            groups = _log(rng, 1, 32)            # (groups of a few values have next to no gradient: eight at least, below)
            case = _gn(kind[3:], _log(rng, 1, 128), _log(rng, 1, 112), _log(rng, 1, 112), groups * _log(rng, 1, 64), groups,
                       rng.choice(ACTS), rng.random() < 0.4)
            if case["h"] * case["w"] * case["channels"] < 8 * groups:
                continue
        elif kind.startswith("adapter"):
            rows = _log(rng, 1, 4096)
            requests = _log(rng, 1, min(rows, 256))
            case = _adapter(kind[8:], rows, _log(rng, 16, 8192), _log(rng, 10, 8192), _log(rng, 1, 64), _log(rng, 1, 64), requests,
                            rng.random() < 0.4, rng.random() < 0.4, rng.random() < 0.2)
        else:
            smallest = _log(rng, 1, 4096)
            case = _grads(rng.choice(("norm", "clip", "step")), _log(rng, 1, 60), smallest, _log(rng, smallest, 6000000),
                          rng.randrange(1 << 20))
        if work(case)["bytes"] <= 6.0e8 and _plain_flops(case) <= 4.0e11:
            return case


def _plain_flops(case):
    """Multiplications and additions of the plain products, which take every row through every adapter."""
    if not case["op"].startswith("adapter"):
        return 0.0
    return 2.0 * case["rows"] * (case["K"] + case["N"]) * case["rank"] * case["adapters"] * (1 if case["op"] == "adapter_fwd" else 2)


def _sizes(case):
    """Element counts of a list of tensors: spread over the logarithm of their range, both ends among them."""
    r = random.Random(case["layout"])
    n = case["tensors"]
    sizes = [_log(r, case["smallest"], case["largest"]) for _ in range(n)]
    sizes[0] = case["largest"]
    sizes[-1] = case["smallest"]
    r.shuffle(sizes)
    return sizes


def _used(case):
    """Adapters that the requests use, on average."""
    n = case["adapters"]
    return n * (1.0 - (1.0 - 1.0 / n) ** case["requests"])


def work(case):
    op = case["op"]
    if op.startswith("gn"):
        x = case["batch"] * case["h"] * case["w"] * case["channels"]
        streams = (2 if op == "gn_fwd" else 3) + (0 if not case["skip"] else 1 if op == "gn_fwd" else 2)
        small = 8 * case["batch"] * case["groups"] + (8 if op == "gn_fwd" else 16) * case["channels"]
        return {"bytes": 4 * x * streams + small, "flops": x * (8 if op == "gn_fwd" else 16)}
    if op.startswith("adapter"):
        M, K, N, r = case["rows"], case["K"], case["N"], case["rank"]
        weights = _used(case) * r * (K + N) * (2 if case["bf16"] else 4)
        flops = 2.0 * M * r * (K + N)
        if op == "adapter_fwd":
            return {"bytes": 4 * M * (K + 2 * N + r) + weights, "flops": flops}
        return {"bytes": 4 * M * (3 * K + N + r) + weights + 4 * case["adapters"] * r * (K + N), "flops": 2 * flops}
    total = sum(_sizes(case))
    return {"bytes": 4 * total * {"grads_norm": 1, "grads_clip": 2, "grads_step": 3}[op], "flops": total * (2 if op == "grads_norm" else 4)}


# ---- the inputs ----------------------------------------------------------------------------------
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _row_adapters(case, seed):
    """Adapter of every row: requests of ragged lengths side by side (or, shuffled, rows in no order); one request in eight has none."""
    r = random.Random(seed)
    cuts = sorted(r.sample(range(1, case["rows"]), case["requests"] - 1)) if case["requests"] > 1 else []
    ends, ids = cuts + [case["rows"]], []
    for q, end in enumerate(ends):
        a = -1 if q % 8 == 7 else r.randrange(case["adapters"])
        ids += [a] * (end - len(ids))
    if case["shuffled"]:
        r.shuffle(ids)
    return torch.tensor(ids, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    s = {"case": case}
    if op.startswith("gn"):
        shape, C, G = (case["batch"], case["h"], case["w"], case["channels"]), case["channels"], case["groups"]
        s["x"] = _randn(gen, *shape) * 2 + _randn(gen, C)            # outputs of a layer: every channel about a mean of its own
        s["gamma"], s["beta"] = 1 + 0.2 * _randn(gen, C), 0.3 * _randn(gen, C)
        s["skip"] = _randn(gen, *shape) if case["skip"] else None
        if op == "gn_bwd":
            s["dy"] = _randn(gen, *shape) * 1e-2
            rows = s["x"].reshape(case["batch"], -1, G, C // G).double()         # what the forward pass kept
            mean = rows.mean((1, 3))
            s["mean"] = mean.float()
            s["invstd"] = (rows.square().mean((1, 3)) - mean.square() + EPS).rsqrt().float()
    elif op.startswith("adapter"):
        M, K, N, r, n = case["rows"], case["K"], case["N"], case["rank"], case["adapters"]
        dtype = torch.bfloat16 if case["bf16"] else torch.float32
        s["rows"] = _row_adapters(case, seed)
        s["X"] = _randn(gen, M, K)
        s["A"] = (_randn(gen, n, r, K) / math.sqrt(K)).to(dtype)
        s["B"] = (_randn(gen, n, r, N) / math.sqrt(r)).to(dtype)
        s["scale"] = 0.5 + torch.rand(n, generator=gen, device="cuda")
        if op == "adapter_fwd":
            s["base"] = _randn(gen, M, N)
        else:
            s["base"], s["dY"] = _randn(gen, M, K) * 1e-2, _randn(gen, M, N) * 1e-2
            s["T"] = _randn(gen, M, r) * (s["rows"] >= 0)[:, None]               # what the forward pass kept
        if own:
            from paper_2002_11151_amd import xbar as xb
            s["plan"] = xb.adapter_plan(s["rows"], n)                            # one for all layers that this batch passes
    else:
        # tensors of their own, gradients of different sizes from layer to layer; the norm is well over what clipping allows
        scales = torch.exp(_randn(gen, case["tensors"])).tolist()
        s["grads"] = [_randn(gen, n) * (scales[i] * 0.1) for i, n in enumerate(_sizes(case))]
        if op == "grads_step":
            s["params"] = [_randn(gen, n) for n in _sizes(case)]
        if own:
            from paper_2002_11151_amd import xbar as xb
            s["grad_list"] = xb.TensorList(s["grads"])
            if op == "grads_step":
                s["param_list"] = xb.TensorList(s["params"])
    return s


# ---- one pass ------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2002_11151_amd import xbar as xb
    case = s["case"]
    op = case["op"]
    if op == "gn_fwd":
        return xb.gn_fwd(s["x"], s["gamma"], s["beta"], case["groups"], EPS, ACTS.index(case["act"]), s["skip"])
    if op == "gn_bwd":
        return xb.gn_bwd(s["x"], s["dy"], s["gamma"], s["beta"], s["mean"], s["invstd"], ACTS.index(case["act"]), s["skip"])
    if op.startswith("adapter"):
        plan = xb.adapter_plan(s["rows"], case["adapters"]) if case["plan"] else s["plan"]
        if op == "adapter_fwd":
            return xb.adapter_fwd(plan, s["base"], s["X"], s["A"], s["B"], s["scale"])
        return xb.adapter_bwd(plan, s["base"], s["dY"], s["X"], s["T"], s["A"], s["B"], s["scale"])
    if op == "grads_norm":
        return xb.grad_norm(s["grad_list"])
    if op == "grads_clip":
        return [xb.grad_clip(s["grad_list"], MAX_NORM)] + s["grads"]
    return [xb.clip_sgd(s["param_list"], s["grad_list"], LR, MAX_NORM)] + s["params"]


def _run_plain(s):
    op = s["case"]["op"]
    if op == "gn_fwd":
        return _plain_gn_fwd(s)
    if op == "gn_bwd":
        return _plain_gn_bwd(s)
    if op == "adapter_fwd":
        return _plain_adapter_fwd(s)
    if op == "adapter_bwd":
        return _plain_adapter_bwd(s)
    return _plain_grads(s)


def _plain_gn_fwd(s):
    case, x = s["case"], s["x"]
    B, G, C = case["batch"], case["groups"], case["channels"]
    rows = x.reshape(B, -1, G, C // G)
    mean = rows.mean((1, 3), keepdim=True)
    d = rows - mean
    invstd = 1.0 / torch.sqrt((d * d).mean((1, 3), keepdim=True) + EPS)
    z = (d * invstd).reshape(x.shape) * s["gamma"] + s["beta"]
    if s["skip"] is not None:
        z = z + s["skip"]
    y = z if case["act"] == "none" else z.clamp(min=0.0) if case["act"] == "relu" else z / (1.0 + torch.exp(-z))
    return y, mean.reshape(B, G), invstd.reshape(B, G)


def _plain_gn_bwd(s):
    case, x, dy = s["case"], s["x"], s["dy"]
    B, G, C = case["batch"], case["groups"], case["channels"]
    mean, invstd = s["mean"][:, None, :, None], s["invstd"][:, None, :, None]
    xhat = ((x.reshape(B, -1, G, C // G) - mean) * invstd).reshape(x.shape)
    g = dy
    if case["act"] == "relu":
        # which side of zero a value lies on decides its whole gradient: in 64 bits
        z = ((x.reshape(B, -1, G, C // G).double() - mean.double()) * invstd.double()).reshape(x.shape) * s["gamma"].double() + s["beta"].double()
        if s["skip"] is not None:
            z = z + s["skip"].double()
        g = torch.where(z > 0, dy, torch.zeros_like(dy))
    elif case["act"] == "silu":
        z = xhat * s["gamma"] + s["beta"]
        if s["skip"] is not None:
            z = z + s["skip"]
        sig = 1.0 / (1.0 + torch.exp(-z))
        g = dy * (sig * (1.0 + z * (1.0 - sig)))
    dbeta, dgamma = g.sum((0, 1, 2)), (g * xhat).sum((0, 1, 2))
    gg = (g * s["gamma"]).reshape(B, -1, G, C // G)
    xh = xhat.reshape(gg.shape)
    dx = invstd * (gg - gg.mean((1, 3), keepdim=True) - xh * (gg * xh).mean((1, 3), keepdim=True))
    out = (dx.reshape(x.shape), dgamma, dbeta)
    return out if s["skip"] is None else out + (g,)


def _plain_mask(s):
    """[rows][adapters rank]: scale of the row's adapter in that adapter's columns, zero elsewhere; and ones in their place."""
    case = s["case"]
    n, r = case["adapters"], case["rank"]
    mine = s["rows"][:, None] == torch.arange(n, device="cuda", dtype=torch.int32)
    ones = mine.float().repeat_interleave(r, dim=1)
    return ones, ones * s["scale"].repeat_interleave(r)


def _plain_adapter_fwd(s):
    case = s["case"]
    n, r, M = case["adapters"], case["rank"], case["rows"]
    A, B = s["A"].float().reshape(n * r, -1), s["B"].float().reshape(n * r, -1)
    ones, scale = _plain_mask(s)
    every = torch.matmul(s["X"], A.t())                   # all adapters' products, of which each row keeps its own
    Y = s["base"] + torch.matmul(every * scale, B)
    return Y, (every * ones).reshape(M, n, r).sum(1)


def _plain_adapter_bwd(s):
    case = s["case"]
    n, r = case["adapters"], case["rank"]
    A, B = s["A"].float().reshape(n * r, -1), s["B"].float().reshape(n * r, -1)
    _, scale = _plain_mask(s)
    dT = torch.matmul(s["dY"], B.t()) * scale
    dX = s["base"] + torch.matmul(dT, A)
    dA = torch.matmul(dT.t().contiguous(), s["X"]).reshape(n, r, -1)
    dB = torch.matmul((s["T"].repeat(1, n) * scale).t().contiguous(), s["dY"]).reshape(n, r, -1)
    return dX, dA, dB


def _plain_grads(s):
    op = s["case"]["op"]
    total = torch.stack([g.double().square().sum() for g in s["grads"]]).sum()       # long sums: 64 bits
    norm = torch.sqrt(total)
    if op == "grads_norm":
        return norm.float().reshape(1)
    c = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm)).float()
    if op == "grads_clip":
        return [norm.float().reshape(1)] + [g.mul_(c) for g in s["grads"]]
    return [norm.float().reshape(1)] + [p.sub_((LR * c) * g) for p, g in zip(s["params"], s["grads"])]


# ---- the definitions in 64 bits ------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    wide = lambda t: None if t is None else t.to(torch.float64)
    if op.startswith("gn"):
        B, C, G = case["batch"], case["channels"], case["groups"]
        x, gamma, beta, skip = (wide(s[k]) for k in ("x", "gamma", "beta", "skip"))
        groups = x.movedim(3, 1).reshape(B, G, -1)                    # one row per sample and group
        if op == "gn_fwd":
            var, mean = torch.var_mean(groups, 2, correction=0)
            invstd = (var + EPS) ** -0.5
        else:
            mean, invstd = wide(s["mean"]), wide(s["invstd"])
        back = lambda t: t.reshape(B, C, case["h"], case["w"]).movedim(1, 3)
        xhat = back((groups - mean[:, :, None]) * invstd[:, :, None])
        z = gamma * xhat + beta + (0.0 if skip is None else skip)
        if op == "gn_fwd":
            y = z if case["act"] == "none" else torch.maximum(z, torch.zeros_like(z)) if case["act"] == "relu" else z * torch.sigmoid(z)
            return y, mean, invstd
        g = wide(s["dy"])
        if case["act"] == "relu":
            g = g * (z > 0)
        elif case["act"] == "silu":
            sig = torch.sigmoid(z)
            g = g * (sig + z * sig * torch.sigmoid(-z))
        share = lambda t: t.movedim(3, 1).reshape(B, G, -1)
        gg, xh = share(gamma * g), share(xhat)
        n = gg.shape[2]
        dx = back(invstd[:, :, None] * (gg - gg.sum(2, keepdim=True) / n - xh * ((gg * xh).sum(2, keepdim=True) / n)))
        out = (dx, (g * xhat).flatten(0, 2).sum(0), g.flatten(0, 2).sum(0))
        return out if skip is None else out + (g,)
    if op.startswith("adapter"):
        X, A, B, scale, base = (wide(s[k]) for k in ("X", "A", "B", "scale", "base"))
        ids = s["rows"].tolist()
        mine = [[m for m, a in enumerate(ids) if a == k] for k in range(case["adapters"])]
        if op == "adapter_fwd":
            T = torch.zeros(case["rows"], case["rank"], dtype=torch.float64, device="cuda")
            Y = base.clone()
            for a, rows in enumerate(mine):
                if rows:
                    at = torch.tensor(rows, device="cuda")
                    T[at] = X[at] @ A[a].t().contiguous()
                    Y[at] += scale[a] * (T[at] @ B[a])
            return Y, T
        T, dY = wide(s["T"]), wide(s["dY"])
        dX, dA, dB = base.clone(), torch.zeros_like(A), torch.zeros_like(B)
        for a, rows in enumerate(mine):
            if rows:
                at = torch.tensor(rows, device="cuda")
                dT = scale[a] * (dY[at] @ B[a].t().contiguous())
                dX[at] += dT @ A[a]
                dA[a] = dT.t().contiguous() @ X[at]
                dB[a] = scale[a] * (T[at].t().contiguous() @ dY[at])
        return dX, dA, dB
    total = 0.0
    for g in s["grads"]:
        total = total + torch.dot(wide(g), wide(g))
    norm = total ** 0.5
    if op == "grads_norm":
        return norm.reshape(1)
    c = torch.clamp(MAX_NORM / norm, max=1.0)
    if op == "grads_clip":
        return [norm.reshape(1)] + [wide(g) * c for g in s["grads"]]
    return [norm.reshape(1)] + [wide(p) - LR * c * wide(g) for p, g in zip(s["params"], s["grads"])]
