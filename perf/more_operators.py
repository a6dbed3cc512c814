"""What is measured of the operators for a worker's training step on rows: layer norm with an activation and a residual,
forward and backward, and the norm of each worker's whole gradient with what clips by it.

A case is one of five kinds, each over G workers at once:

* ``forward``   s = x + r (stored in x's type; s = x without a residual);  y = act(gamma (s - mean) rstd + beta), mean and rstd
                of each row of C values, rows at a stride of their own.
* ``backward``  the gradients of s, gamma and beta from that of y, the residual's own added to the first; ReLU's derivative goes
                by the stored y > 0, as everywhere in this library.
* ``norm``      sqrt(sum g^2) of each worker over all of its tensors.
* ``clip``      the same, and every gradient times min(1, max_norm / norm), into another buffer's places (a pass would find its
                own result clipped already, were it in place).
* ``update``    the same norm, and the local momentum step with the gradient so clipped: g' = f g + wd w;  u = m u + g';
                w -= lr (g' + m u or u), and w's bf16 copy.

``own`` false: the same in plain torch, 32 bits, sums of squares in 64; ``own`` true: the library's calls.
"""
import math
import random

import torch

own = False

EPS, LR, MOMENTUM, DECAY = 1e-5, 0.02, 0.9, 5e-4

# ------------------------------------------------------------------------------------- the cases


def _rows(kind, G, R, C, x="bf16", y="bf16", act="none", residual=False, pad=False):
    """pad: rows start at multiples of 8 values, as the dense layers' activations do; else one behind another."""
    return dict(kind=kind, G=G, R=R, C=C, x=x, y=y, act=act, residual=residual, pad=pad)


def _grads(kind, G, tensors, g="fp32", ratio=0.3, arena=True, **kw):
    """tensors: ``resnet20``, ``dense:<widths>`` or ``ragged:<number>:<mean size>:<seed>``.  arena: they stand in one buffer, a
    worker's one behind another, each from a multiple of 64 values on (what ``clip`` writes always does); else a tensor of
    [G][values] each.  ratio: of
    max_norm to the norm that the values' distribution leads to expect (never near 1, where a rounding decides)."""
    return dict(kind=kind, G=G, tensors=tensors, g=g, ratio=ratio, arena=arena, **kw)


def listed():
    return [
        # one worker's evaluation batch, odd in both: latency
        dict(_rows("forward", 1, 50, 777, "fp32", "fp32", "silu"), name="forward_small_odd"),
        # a hidden layer of the 4096-wide MLP at the paper's 16 workers x 128: fp32 products to the next layer's bf16 operand
        dict(_rows("forward", 16, 128, 4096, "fp32", "bf16", "relu"), name="forward_mlp4096"),
        # long batches of wide rows with a residual stream in bf16: bandwidth
        dict(_rows("forward", 4, 8192, 2048, residual=True), name="forward_residual"),
        # the gradients of that hidden layer
        dict(_rows("backward", 16, 128, 4096, "fp32", "bf16", "relu"), name="backward_mlp4096"),
        # ... and of the residual stream
        dict(_rows("backward", 4, 8192, 2048, residual=True), name="backward_residual"),
        # an odd width in rows of whole vectors, SiLU, an odd number of workers and rows
        dict(_rows("backward", 3, 517, 1531, "bf16", "bf16", "silu", pad=True), name="backward_odd"),
        # ResNet-20's gradients of 16 workers, 59 tensors of 10 to 36,864 values: latency
        dict(_grads("norm", 16, "resnet20"), name="norm_resnet20"),
        # the 4096-wide MLP's of 8 workers: bandwidth
        dict(_grads("norm", 8, "dense:4096,4096,4096,100"), name="norm_mlp4096"),
        # one worker's 300 tensors of any size in bf16, as autograd leaves them: the table of tensors
        dict(_grads("clip", 1, "ragged:300:40000:5", "bf16", arena=False, out="bf16"), name="clip_ragged"),
        # the 1024-wide network's of 16 workers, clipped into bf16 for a direction's products
        dict(_grads("clip", 16, "dense:1024,1024,1024,10", out="bf16"), name="clip_mlp1024"),
        # ResNet-20's step, no decay for the last 1,376 (BatchNorm's) values: latency
        dict(_grads("update", 16, "resnet20", nesterov=True, ratio=3.0), name="update_resnet20"),
        # the 4096-wide MLP's step: bandwidth
        dict(_grads("update", 8, "dense:4096,4096,4096,100", nesterov=True), name="update_mlp4096"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 7e12, w["flops"] / 8e13)


def draw(rng):
    kind = rng.choice(("forward", "forward", "backward", "backward", "norm", "clip", "update"))
    top = max(_cost(c) for c in listed() if c["kind"] == kind)
    while True:
        if kind in ("forward", "backward"):
            x = rng.choice(("bf16", "fp32"))
            c = _rows(kind, _log_int(rng, 1, 32), _log_int(rng, 1, 30000), _log_int(rng, 4, 20000), x,
                      x if rng.random() < 0.6 else rng.choice(("bf16", "fp32")), rng.choice(("none", "relu", "silu")),
                      rng.random() < 0.5, rng.random() < 0.6)
        else:
            form = rng.choice(("resnet20", "dense", "ragged"))
            if form == "dense":
                form += ":" + ",".join(str(_log_int(rng, 10, 4096)) for _ in range(rng.randint(2, 5)))
            elif form == "ragged":
                form += f":{_log_int(rng, 1, 700)}:{_log_int(rng, 4, 200000)}:{rng.randrange(1000)}"
            c = _grads(kind, _log_int(rng, 1, 64), form, rng.choice(("fp32", "fp32", "bf16")),
                       rng.choice((0.05, 0.3, 0.7, 1.5, 4.0)), rng.random() < 0.6)
            if kind == "clip":
                c["out"] = rng.choice(("fp32", "bf16"))
            if kind == "update":
                c["nesterov"] = rng.random() < 0.6
        if _cost(c) <= top:
            return c


def _sizes(case):
    """The numbers of values of a worker's tensors."""
    form, _, rest = case["tensors"].partition(":")
    if form == "dense":
        w = [int(v) for v in rest.split(",")]
        return [n for i, o in zip(w, w[1:]) for n in (i * o, o)]
    if form == "ragged":
        count, mean, seed = (int(v) for v in rest.split(":"))
        rng = random.Random(seed)
        return [max(1, int(rng.expovariate(1 / mean))) for _ in range(count)]
    convs = [(3, 16)] + [(16, 16)] * 6 + [(16, 32)] + [(32, 32)] * 5 + [(32, 64)] + [(64, 64)] * 5
    return [9 * i * o for i, o in convs] + [640, 10] + [o for _, o in convs for _ in range(2)]


def _layout(case):
    """(offsets of a worker's tensors in an arena, its values with their padding)."""
    offsets, at = [], 0
    for n in _sizes(case):
        offsets.append(at)
        at += (n + 63) // 64 * 64
    return offsets, at


def _ld(case):
    return (case["C"] + 7) // 8 * 8 if case["pad"] else case["C"]


# --------------------------------------------------------------------------- inputs from the seed

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, G, e = case["kind"], case["G"], dict(device="cuda")
    s = dict(case=case)
    if kind in ("forward", "backward"):
        R, C, ld, xt, yt = case["R"], case["C"], _ld(case), _TYPES[case["x"]], _TYPES[case["y"]]
        # a layer's outputs: columns and rows of different sizes, with a mean
        x = (_randn(g, G, R, ld) * (0.5 + torch.rand(G, R, 1, generator=g, **e)) + _randn(g, 1, 1, ld)).to(xt)
        s.update(x=x, gamma=1 + 0.2 * _randn(g, G, C), beta=0.2 * _randn(g, G, C))
        y, mean, rstd = torch.zeros(G, R, ld, dtype=yt, **e), torch.empty(G, R, **e), torch.empty(G, R, **e)
        if kind == "forward":
            s.update(y=y, mean=mean, rstd=rstd)
            if case["residual"]:
                s.update(r=_randn(g, G, R, ld).to(xt), s=torch.zeros_like(x))
        else:
            # the forward's results, and gradients of a mean over the rows
            y[..., :C], s["mean"], s["rstd"] = _plain_rows(case, s, x[..., :C].float())
            s.update(y=y if case["act"] == "relu" else None, dy=(_randn(g, G, R, ld) / R).to(yt), dx=torch.zeros_like(x),
                     dgamma=torch.empty(G, C, **e), dbeta=torch.empty(G, C, **e))
            if case["residual"]:
                s["ds"] = (_randn(g, G, R, ld) / R).to(xt)
        return s
    # gradients: tensors of different sizes of values, a few of a tensor's values zero (dead units)
    sizes, (offsets, total), gt = _sizes(case), _layout(case), _TYPES[case["g"]]
    rng = random.Random(int(seed))
    scales = [10 ** rng.uniform(-4, -2) for _ in sizes]
    s["max_norm"] = case["ratio"] * math.sqrt(sum(0.9 * n * v * v for n, v in zip(sizes, scales)))

    def fill(n, scale):
        return (scale * _randn(g, G, n) * (torch.rand(G, n, generator=g, **e) < 0.9)).to(gt)

    def views(buf):
        return [buf[:, o:o + n] for o, n in zip(offsets, sizes)]

    if case["arena"] or kind == "update":  # the update takes a worker's values as one block
        s["g"] = torch.zeros(G, total, dtype=gt, **e)
        grads = views(s["g"])
        for t, v in zip(grads, scales):
            t.copy_(fill(t.shape[1], v))
    else:
        grads = [fill(n, v) for n, v in zip(sizes, scales)]
    s.update(grads=grads, norm=torch.empty(G, **e))
    if kind == "clip":
        s["out"] = torch.zeros(G, total, dtype=_TYPES[case["out"]], **e)
        s["outs"] = views(s["out"])
    if kind == "update":
        s.update(w=0.05 * _randn(g, G, total), u=0.005 * _randn(g, G, total),
                 wb=torch.empty(G, total, dtype=torch.bfloat16, **e),
                 # (weight decay is not for BatchNorm's parameters, which stand last)
                 decay_end=offsets[21] if case["tensors"] == "resnet20" else total)
    if own:
        import paper_1808_07217_gb300 as lsgd

        # a program's gradients keep their places: it describes them once
        s["list"] = lsgd.lsgd_tensors_create(grads, s.get("outs"))
    return s


# -------------------------------------------------------------------------------- the plain forms


def _plain_rows(case, s, x):
    """y in its type, mean and rstd of float rows x [G][R][C]."""
    mean = x.mean(-1, keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(-1, keepdim=True) + EPS)
    z = (x - mean) * rstd * s["gamma"][:, None] + s["beta"][:, None]
    y = torch.relu(z) if case["act"] == "relu" else z / (1 + torch.exp(-z)) if case["act"] == "silu" else z
    return y.to(_TYPES[case["y"]]), mean[..., 0], rstd[..., 0]


def _plain_forward(case, s):
    x, C = s["x"], case["C"]
    out = {}
    if case["residual"]:
        out["s"] = x = (x[..., :C].float() + s["r"][..., :C].float()).to(x.dtype)
    out["y"], out["mean"], out["rstd"] = _plain_rows(case, s, x[..., :C].float())
    return out


def _plain_backward(case, s):
    C = case["C"]
    xh = (s["x"][..., :C].float() - s["mean"][..., None]) * s["rstd"][..., None]
    dz, gamma = s["dy"][..., :C].float(), s["gamma"][:, None]
    if case["act"] == "relu":
        dz = dz * (s["y"][..., :C] > 0)
    elif case["act"] == "silu":
        z = xh * gamma + s["beta"][:, None]
        sg = 1 / (1 + torch.exp(-z))
        dz = dz * sg * (1 + z * (1 - sg))
    t = dz * gamma
    dx = s["rstd"][..., None] * (t - t.mean(-1, keepdim=True) - xh * (t * xh).mean(-1, keepdim=True))
    if case["residual"]:
        dx = dx + s["ds"][..., :C].float()
    return dict(dx=dx.to(s["x"].dtype), dgamma=(dz * xh).sum(1), dbeta=dz.sum(1))


def _plain_norm(s):
    sums = [t.float().square().sum(1, dtype=torch.float64) for t in s["grads"]]
    norm = torch.stack(sums).sum(0).sqrt()
    return norm.float(), torch.clamp(s["max_norm"] / norm, max=1.0).float()[:, None]


# ------------------------------------------------------------------------------------- one pass


def run(state):
    s, case = state, state["case"]
    kind, C = case["kind"], case.get("C")
    if own:
        import paper_1808_07217_gb300 as lsgd

        if kind in ("forward", "backward"):
            act = {"none": lsgd.ACT_NONE, "relu": lsgd.ACT_RELU, "silu": lsgd.ACT_SILU}[case["act"]]
            kw = dict(act=act, x_ld=_ld(case), y_ld=_ld(case))
            shape = (case["G"], case["R"], C)
            if kind == "forward":
                lsgd.lsgd_layernorm_forward(s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], *shape, r=s.get("r"),
                                            s=s.get("s"), eps=EPS, **kw)
                out = dict(y=s["y"][..., :C], mean=s["mean"], rstd=s["rstd"])
                return dict(out, s=s["s"][..., :C]) if case["residual"] else out
            lsgd.lsgd_layernorm_backward(s["x"], s["y"], s["dy"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["dx"],
                                         s["dgamma"], s["dbeta"], *shape, ds=s.get("ds"), **kw)
            return dict(dx=s["dx"][..., :C], dgamma=s["dgamma"], dbeta=s["dbeta"])
        if kind == "norm":
            lsgd.lsgd_gradient_norm(s["list"], s["norm"])
            return dict(norm=s["norm"])
        if kind == "clip":
            lsgd.lsgd_gradient_clip(s["list"], s["norm"], s["max_norm"])
            return dict(norm=s["norm"], out=s["out"])
        lsgd.lsgd_gradient_norm(s["list"], s["norm"])
        lsgd.lsgd_clipped_update(s["w"], s["u"], s["g"], s["wb"], case["G"], s["w"].shape[1], s["norm"], s["max_norm"], LR,
                                 momentum=MOMENTUM, nesterov=case["nesterov"], weight_decay=DECAY, decay_end=s["decay_end"])
        return dict(norm=s["norm"], w=s["w"], u=s["u"], wb=s["wb"])
    if kind == "forward":
        return _plain_forward(case, s)
    if kind == "backward":
        return _plain_backward(case, s)
    norm, factor = _plain_norm(s)
    if kind == "norm":
        return dict(norm=norm)
    if kind == "clip":
        for t, o in zip(s["grads"], s["outs"]):
            o.copy_(t.float() * factor)
        return dict(norm=norm, out=s["out"])
    w, u, end = s["w"], s["u"], s["decay_end"]
    g = s["g"].float() * factor
    g[:, :end] += DECAY * w[:, :end]
    u.mul_(MOMENTUM).add_(g)
    w.sub_(LR * (g + MOMENTUM * u if case["nesterov"] else u))
    return dict(norm=norm, w=w, u=u, wb=w.bfloat16())


# ------------------------------------------------------------------- bytes and operations of one


def work(case):
    size = {"bf16": 2, "fp32": 4}
    kind, G = case["kind"], case["G"]
    if kind in ("forward", "backward"):
        x, y, n = size[case["x"]], size[case["y"]], G * case["R"] * case["C"]
        params, stats = 8 * G * case["C"], 8 * G * case["R"]
        if kind == "forward":
            return {"bytes": n * (x + y + (2 * x if case["residual"] else 0)) + params + stats, "flops": 10 * n}
        each = 2 * x + y + (y if case["act"] == "relu" else 0) + (x if case["residual"] else 0)
        return {"bytes": n * each + 2 * params + stats, "flops": 20 * n}
    n, g = G * sum(_sizes(case)), size[case["g"]]
    if kind == "norm":
        return {"bytes": n * g + 4 * G, "flops": 2 * n}
    if kind == "clip":
        return {"bytes": n * (g + size[case["out"]]) + 4 * G, "flops": 3 * n}
    n = G * _layout(case)[1]
    return {"bytes": n * (g + 18) + 4 * G, "flops": 11 * n}


# --------------------------------------------------------------------- the definitions in 64 bits


def exact(case, seed):
    global own
    kept, own = own, False  # (the inputs alone, without the library's list)
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    kind, G = case["kind"], case["G"]
    out = {}
    if kind in ("forward", "backward"):
        C, Rn = case["C"], case["R"]
        names = ["y", "mean", "rstd"] + (["s"] if case["residual"] else []) if kind == "forward" else ["dx", "dgamma", "dbeta"]
        parts = {k: [] for k in names}
        for k in range(G):  # a worker at a time
            d = {n: v[k].double() for n, v in s.items() if torch.is_tensor(v)}
            x, ga, be = d["x"][:, :C], d["gamma"], d["beta"]
            if kind == "forward":
                if case["residual"]:
                    sums = x + d["r"][:, :C]
                    parts["s"].append(sums)
                    x = sums.to(s["x"].dtype).double()  # what is stored is what is normalised
                var, mean = torch.var_mean(x, -1, correction=0)
                rstd = (var + EPS) ** -0.5
                z = torch.addcmul(be, (x - mean[:, None]) * rstd[:, None], ga)
                y = z.clamp(min=0) if case["act"] == "relu" else z * torch.sigmoid(z) if case["act"] == "silu" else z
                for n, v in (("y", y), ("mean", mean), ("rstd", rstd)):
                    parts[n].append(v)
                continue
            xh = (x - d["mean"][:, None]) * d["rstd"][:, None]
            dz = d["dy"][:, :C]
            if case["act"] == "relu":
                dz = torch.where(d["y"][:, :C] > 0, dz, 0.0)
            elif case["act"] == "silu":
                z = torch.addcmul(be, xh, ga)
                sg = torch.sigmoid(z)
                dz = dz * (sg + z * sg * (1 - sg))
            parts["dgamma"].append(torch.einsum("rc,rc->c", dz, xh))
            parts["dbeta"].append(dz.sum(0))
            m1, m2 = (dz @ ga) / C, torch.einsum("rc,rc,c->r", dz, xh, ga) / C
            dx = (dz * ga - m1[:, None] - xh * m2[:, None]) * d["rstd"][:, None]
            parts["dx"].append(dx + d["ds"][:, :C] if case["residual"] else dx)
        out = {k: torch.stack(v) for k, v in parts.items()}
        return {k: out[k] for k in names}
    norm = torch.zeros(G, dtype=torch.float64, device="cuda")
    for t in s["grads"]:
        norm = torch.hypot(norm, torch.linalg.vector_norm(t.double(), dim=1))
    if kind == "norm":
        return dict(norm=norm)
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    if kind == "clip":
        clipped = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        for t, at in zip(s["grads"], _layout(case)[0]):
            clipped[:, at:at + t.shape[1]] = t.double() * factor[:, None]
        return dict(norm=norm, out=clipped)
    w, u = torch.empty_like(s["w"], dtype=torch.float64), torch.empty_like(s["w"], dtype=torch.float64)
    decay = torch.zeros(s["w"].shape[1], dtype=torch.float64, device="cuda")
    decay[:s["decay_end"]] = DECAY
    for k in range(G):
        old = s["w"][k].double()
        step = s["g"][k].double() * factor[k] + decay * old
        u[k] = MOMENTUM * s["u"][k].double() + step
        w[k] = old - LR * (step + MOMENTUM * u[k] if case["nesterov"] else u[k])
    return dict(norm=norm, w=w, u=u, wb=w)
