"""What is measured of two pairs of operators for one worker's training step: a normalisation that keeps
no statistics from step to step (group norm with an activation, channels last, forward and backward)
and an update whose direction is the momentum with its singular values brought near one.

A case is one of four kinds, each over G workers' tensors at once:

* ``direction``  u = m u + g;  x = g + m u (Nesterov) or u;  X = x / ||x||_F;  STEPS times
                 X = a X + (b A + c A A) X with A = X X^T;  o = X in bf16.  Outputs u and o.
* ``update``     w = (1 - lr wd) w - lr scale o and its bf16 copy.
* ``forward``    y = act(gamma (x - mean) rstd + beta), mean and rstd per image and group of channels.
* ``backward``   the gradients of x, gamma and beta from that of y; ReLU's derivative goes by the stored
                 y > 0, as everywhere in this library.

``own`` false: the same in plain torch, 32 bits; ``own`` true: the library's calls.
"""
import math

import torch

own = False

STEPS, MOMENTUM = 5, 0.95
A, B, C = 3.4445, -4.7750, 2.0315  # the published quintic's coefficients (Jordan et al. 2024)
LR, DECAY, EPS = 0.02, 0.01, 1e-5

# ------------------------------------------------------------------------------------- the cases


def _direction(G, rows, cols, grad="fp32", nesterov=True, batch=128):
    return dict(kind="direction", G=G, rows=rows, cols=cols, grad=grad, nesterov=nesterov, batch=batch)


def _update(G, rows, cols, shadow=True):
    return dict(kind="update", G=G, rows=rows, cols=cols, shadow=shadow)


def _norm(kind, G, B, P, C, groups, act, x="bf16", y="bf16"):
    return dict(kind=kind, G=G, B=B, P=P, C=C, groups=groups, act=act, x=x, y=y)


def listed():
    return [
        # ResNet-20's first-stage convolution weights (16 x 3 x 3 x 16) of 16 workers: latency
        dict(_direction(16, 16, 144), name="direction_conv16"),
        # the 100-class layer of the 4096-wide MLP: few rows, odd against every tile, a long product
        dict(_direction(16, 100, 4096), name="direction_head100"),
        # the hidden layer of the 1024-wide MLP at the paper's 16 workers
        dict(_direction(16, 1024, 1024), name="direction_mlp1024"),
        # a layer with more outputs than inputs, odd in both, gradients kept in bf16, few samples
        dict(_direction(5, 1031, 777, grad="bf16", nesterov=False, batch=50), name="direction_tall_odd"),
        # a hidden layer of the 4096-wide MLP, four workers: bound by the products
        dict(_direction(4, 4096, 4096), name="direction_mlp4096"),
        # applying the direction to third-stage convolution weights (64 x 3 x 3 x 64): latency
        dict(_update(16, 64, 576), name="update_conv64"),
        # ... and to a 4096-wide layer of 16 workers: bandwidth
        dict(_update(16, 4096, 4096), name="update_mlp4096"),
        # one worker's evaluation batch at the last stage: latency
        dict(_norm("forward", 1, 16, 64, 64, 8, "relu"), name="forward_small"),
        # ResNet-20's first stage at 16 workers x 128 images, fp32 convolution outputs to bf16
        dict(_norm("forward", 16, 128, 1024, 16, 4, "relu", x="fp32"), name="forward_stage1"),
        # few large images, ten channels to a group, an odd number of positions
        dict(_norm("forward", 2, 4, 127 * 129, 320, 32, "silu"), name="forward_large"),
        # the backward of that first stage
        dict(_norm("backward", 16, 128, 1024, 16, 4, "relu", x="fp32"), name="backward_stage1"),
        # fp32 throughout, odd sizes everywhere
        dict(_norm("backward", 3, 5, 37 * 41, 90, 9, "silu", x="fp32", y="fp32"), name="backward_odd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 7e12, w["flops"] / 2e15)


def draw(rng):
    kind = rng.choice(("direction", "direction", "update", "forward", "backward"))
    top = max(_cost(c) for c in listed() if c["kind"] == kind)
    while True:
        if kind == "direction":
            c = _direction(_log_int(rng, 1, 64), _log_int(rng, 4, 4096), _log_int(rng, 4, 4096),
                           rng.choice(("fp32", "fp32", "bf16")), rng.random() < 0.7, _log_int(rng, 16, 256))
        elif kind == "update":
            c = _update(_log_int(rng, 1, 64), _log_int(rng, 4, 4096), _log_int(rng, 4, 4096), rng.random() < 0.8)
        else:
            groups = rng.choice((1, 2, 3, 4, 8, 16, 32))
            x = rng.choice(("bf16", "bf16", "fp32"))
            c = _norm(kind, _log_int(rng, 1, 16), _log_int(rng, 1, 128), _log_int(rng, 4, 20000),
                      groups * _log_int(rng, 1, 512 // groups), groups, rng.choice(("none", "relu", "silu")),
                      x, x if rng.random() < 0.7 else rng.choice(("bf16", "fp32")))
        if _cost(c) <= top:
            return c


# --------------------------------------------------------------------------- inputs from the seed

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, G = case["kind"], case["G"]
    s = dict(case=case)
    if kind == "direction":
        rows, cols, n = case["rows"], case["cols"], case["batch"]

        def gradient(k):  # dZ^T act over k mini-batches, as a dense layer's weight gradient is
            dz = _randn(g, G, k * n, rows) / n
            act = torch.relu(_randn(g, G, k * n, cols))
            return torch.bmm(dz.transpose(1, 2), act)

        s.update(g=gradient(1).to(_TYPES[case["grad"]]), u=1.5 * gradient(3),
                 o=torch.empty(G, rows, cols, device="cuda", dtype=torch.bfloat16))
    elif kind == "update":
        rows, cols = case["rows"], case["cols"]
        w = math.sqrt(2.0 / cols) * _randn(g, G, rows, cols)
        o = (_randn(g, G, rows, cols) / math.sqrt(max(rows, cols))).bfloat16()
        s.update(w=w, o=o, wb=torch.empty_like(o) if case["shadow"] else None)
    else:
        N, P, ch, groups = G * case["B"], case["P"], case["C"], case["groups"]
        xt, yt, e = _TYPES[case["x"]], _TYPES[case["y"]], dict(device="cuda")
        x = (_randn(g, N, P, ch) * (0.5 + torch.rand(N, 1, ch, generator=g, **e)) + _randn(g, 1, 1, ch)).to(xt)
        s.update(x=x, gamma=1 + 0.2 * _randn(g, G, ch), beta=0.2 * _randn(g, G, ch))
        if kind == "forward":
            s.update(y=torch.empty(N, P, ch, dtype=yt, **e), mean=torch.empty(N, groups, **e),
                     rstd=torch.empty(N, groups, **e))
        else:
            y, mean, rstd = _plain_forward(case, s)
            s.update(y=y, mean=mean, rstd=rstd, dy=(_randn(g, N, P, ch) / case["B"]).to(yt),
                     dx=torch.empty_like(x), dgamma=torch.empty(G, ch, **e), dbeta=torch.empty(G, ch, **e))
    return s


# -------------------------------------------------------------------------------- the plain forms


def _plain_direction(case, s):
    g, u = s["g"].float(), s["u"]
    u.mul_(MOMENTUM).add_(g)
    x = g + MOMENTUM * u if case["nesterov"] else u
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt()
    X = torch.where(norm > 0, x / norm, 0.0).float()
    wide = case["rows"] <= case["cols"]
    for _ in range(STEPS):
        if wide:
            M = torch.bmm(X, X.transpose(1, 2))
            X = A * X + torch.bmm(B * M + C * torch.bmm(M, M), X)
        else:
            M = torch.bmm(X.transpose(1, 2), X)
            X = A * X + torch.bmm(X, B * M + C * torch.bmm(M, M))
    return u, X.bfloat16()


def _affine(case, s, by_group):
    """gamma or beta of every image's worker, as [N][1][groups][channels of a group]."""
    return by_group.repeat_interleave(case["B"], 0).reshape(-1, 1, case["groups"], case["C"] // case["groups"])


def _grouped(case, t):
    return t.float().reshape(t.shape[0], case["P"], case["groups"], -1)


def _plain_forward(case, s):
    x = _grouped(case, s["x"])
    mean = x.mean((1, 3), keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean((1, 3), keepdim=True) + EPS)
    z = (x - mean) * rstd * _affine(case, s, s["gamma"]) + _affine(case, s, s["beta"])
    y = torch.relu(z) if case["act"] == "relu" else z / (1 + torch.exp(-z)) if case["act"] == "silu" else z
    return y.reshape(s["x"].shape).to(_TYPES[case["y"]]), mean[:, 0, :, 0], rstd[:, 0, :, 0]


def _plain_backward(case, s):
    N = s["x"].shape[0]
    mean, rstd = (s[k].reshape(N, 1, -1, 1) for k in ("mean", "rstd"))
    gamma = _affine(case, s, s["gamma"])
    xh = (_grouped(case, s["x"]) - mean) * rstd
    dz = _grouped(case, s["dy"])
    if case["act"] == "relu":
        dz = dz * (_grouped(case, s["y"]) > 0)
    elif case["act"] == "silu":
        z = xh * gamma + _affine(case, s, s["beta"])
        sg = 1 / (1 + torch.exp(-z))
        dz = dz * sg * (1 + z * (1 - sg))
    each = lambda t: t.sum(1).reshape(case["G"], case["B"], -1).sum(1)  # noqa: E731
    dgamma, dbeta = each(dz * xh), each(dz)
    dxh = dz * gamma
    dx = rstd * (dxh - dxh.mean((1, 3), keepdim=True) - xh * (dxh * xh).mean((1, 3), keepdim=True))
    return dx.reshape(s["x"].shape).to(s["x"].dtype), dgamma, dbeta


# ------------------------------------------------------------------------------------- one pass


def run(state):
    s, case = state, state["case"]
    kind, G = case["kind"], case["G"]
    if own:
        import paper_1808_07217_gb300 as lsgd

        if kind == "direction":
            lsgd.lsgd_orthogonal_direction(s["u"], s["g"], s["o"], G, case["rows"], case["cols"],
                                           momentum=MOMENTUM, nesterov=case["nesterov"], steps=STEPS)
            return dict(u=s["u"], o=s["o"])
        if kind == "update":
            rows, cols = case["rows"], case["cols"]
            lsgd.lsgd_direction_update(s["w"], s["o"], s["wb"], G, rows * cols, LR,
                                       scale=math.sqrt(max(1.0, rows / cols)), weight_decay=DECAY)
            return dict(w=s["w"], wb=s["wb"])
        act = {"none": lsgd.ACT_NONE, "relu": lsgd.ACT_RELU, "silu": lsgd.ACT_SILU}[case["act"]]
        shape = (G, case["B"], case["P"], case["C"], case["groups"])
        if kind == "forward":
            lsgd.lsgd_groupnorm_forward(s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], *shape,
                                        act=act, eps=EPS)
            return dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
        lsgd.lsgd_groupnorm_backward(s["x"], s["y"], s["dy"], s["gamma"], s["beta"], s["mean"], s["rstd"],
                                     s["dx"], s["dgamma"], s["dbeta"], *shape, act=act)
        return dict(dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
    if kind == "direction":
        u, o = _plain_direction(case, s)
        return dict(u=u, o=o)
    if kind == "update":
        w = s["w"]
        w.mul_(1 - LR * DECAY).sub_(s["o"].float() * (LR * math.sqrt(max(1.0, case["rows"] / case["cols"]))))
        return dict(w=w, wb=w.bfloat16() if case["shadow"] else None)
    if kind == "forward":
        y, mean, rstd = _plain_forward(case, s)
        return dict(y=y, mean=mean, rstd=rstd)
    dx, dgamma, dbeta = _plain_backward(case, s)
    return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)


# ------------------------------------------------------------------- bytes and operations of one


def work(case):
    kind, G = case["kind"], case["G"]
    if kind == "direction":
        n, m = sorted((case["rows"], case["cols"]))
        # g in, u in and out, o out; of the two symmetric products one triangle, the third in full
        step = n * (n + 1) * m + n * (n + 1) * n + 2 * n * n * m
        return {"bytes": G * n * m * ((4 if case["grad"] == "fp32" else 2) + 8 + 2), "flops": G * STEPS * step}
    if kind == "update":
        n = G * case["rows"] * case["cols"]
        return {"bytes": n * (4 + 2 + 4 + (2 if case["shadow"] else 0)), "flops": 3 * n}
    size = {"bf16": 2, "fp32": 4}
    x, y, N = size[case["x"]], size[case["y"]], G * case["B"]
    n, params, stats = N * case["P"] * case["C"], 8 * G * case["C"], 8 * N * case["groups"]
    if kind == "forward":
        return {"bytes": n * (x + y) + params + stats, "flops": 10 * n}
    return {"bytes": n * (2 * x + y * (2 if case["act"] == "relu" else 1)) + 2 * params + stats, "flops": 20 * n}


# --------------------------------------------------------------------- the definitions in 64 bits


def exact(case, seed):
    s, kind, G = prepare(case, seed), case["kind"], case["G"]
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
    if kind == "direction":
        u = MOMENTUM * d["u"] + d["g"]
        out = torch.empty_like(u)
        for k in range(G):
            X = d["g"][k] + MOMENTUM * u[k] if case["nesterov"] else u[k]
            X = X if case["rows"] <= case["cols"] else X.t()
            X = X / torch.linalg.vector_norm(X)
            for _ in range(STEPS):  # Horner's form of the quintic
                gram = X @ X.t()
                X = A * X + gram @ (B * X + C * (gram @ X))
            out[k] = X if case["rows"] <= case["cols"] else X.t()
        return dict(u=u, o=out)
    if kind == "update":
        w = d["w"] - LR * (DECAY * d["w"] + math.sqrt(max(1.0, case["rows"] / case["cols"])) * d["o"])
        return dict(w=w, wb=w if case["shadow"] else None)
    P, groups = case["P"], case["groups"]
    D, Bn = case["C"] // groups, case["B"]
    out = {k: [] for k in (("y", "mean", "rstd") if kind == "forward" else ("dx", "dgamma", "dbeta"))}
    for k in range(G):
        at = slice(k * Bn, (k + 1) * Bn)
        x = d["x"][at].reshape(Bn, P, groups, D).permute(0, 2, 1, 3).reshape(Bn, groups, P * D)
        back = lambda t: t.reshape(Bn, groups, P, D).permute(0, 2, 1, 3).reshape(Bn, P, groups * D)  # noqa: E731
        if kind == "forward":
            var, mean = torch.var_mean(x, -1, correction=0)
            rstd = (var + EPS) ** -0.5
            z = back((x - mean[..., None]) * rstd[..., None]) * d["gamma"][k] + d["beta"][k]
            y = z.clamp(min=0) if case["act"] == "relu" else z * torch.sigmoid(z) if case["act"] == "silu" else z
            for name, v in (("y", y), ("mean", mean), ("rstd", rstd)):
                out[name].append(v)
            continue
        rstd = d["rstd"][at][..., None]
        xh = back((x - d["mean"][at][..., None]) * rstd)
        dz = d["dy"][at]
        if case["act"] == "relu":
            dz = torch.where(d["y"][at] > 0, dz, 0.0)
        elif case["act"] == "silu":
            z = xh * d["gamma"][k] + d["beta"][k]
            sg = torch.sigmoid(z)
            dz = dz * (sg + z * sg * (1 - sg))
        out["dgamma"].append((dz * xh).sum((0, 1)))
        out["dbeta"].append(dz.sum((0, 1)))
        t = (dz * d["gamma"][k]).reshape(Bn, P, groups, D).permute(0, 2, 1, 3).reshape(Bn, groups, P * D)
        h = xh.reshape(Bn, P, groups, D).permute(0, 2, 1, 3).reshape(Bn, groups, P * D)
        out["dx"].append(back(rstd * (t - t.mean(-1, keepdim=True) - h * (t * h).mean(-1, keepdim=True))))
    join = torch.stack if kind == "backward" else torch.cat
    return {k: torch.cat(v) if k == "dx" else join(v) for k, v in out.items()}
