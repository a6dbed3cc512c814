"""Overlapping tensors are refused, whichever they are; parameters that stand between each other's are not."""
import ctypes

import pytest

BIG = 1 << 32
NAMES = ["x", "gamma", "beta", "y", "mean", "rstd", "dy", "dx", "dgamma", "dbeta", "ws"]


def _sizes(G, B, P, C, groups, par_gs, need):
    n, span, ns = G * B * P * C, 4 * ((G - 1) * par_gs + C), 4 * G * B * groups
    return dict(x=2 * n, y=4 * n, dy=4 * n, dx=2 * n, gamma=span, beta=span, dgamma=span, dbeta=span, mean=ns, rstd=ns, ws=need)


def _call(fn, shape, par_gs, act=1, **at):
    """The C call with addresses that are never used: each call here is refused, or would be without a GPU."""
    from paper_1808_07217_gb300 import _build

    _build.build()
    import paper_1808_07217_gb300 as L

    G, B, P, C, groups = shape
    need = L.lsgd_groupnorm_workspace(*shape, fn == "backward")
    a = {k: (i + 1) * BIG for i, k in enumerate(NAMES)}
    sizes = _sizes(*shape, par_gs, need)
    a.update({k: v(a, sizes) if callable(v) else v for k, v in at.items()})
    vp = lambda k: ctypes.c_void_p(a[k])  # noqa: E731
    if fn == "forward":
        s = L.lib().lsgd_groupnorm_forward(vp("x"), L.BF16, vp("gamma"), vp("beta"), par_gs, vp("y"), L.FP32, vp("mean"), vp("rstd"),
                                           G, B, P, C, groups, 1e-5, act, vp("ws"), need, None)
    else:
        s = L.lib().lsgd_groupnorm_backward(vp("x"), L.BF16, vp("y"), vp("dy"), L.FP32, vp("gamma"), vp("beta"), par_gs, vp("mean"),
                                            vp("rstd"), vp("dx"), vp("dgamma"), vp("dbeta"), G, B, P, C, groups, act, vp("ws"),
                                            need, None)
    return s, L.lsgd_last_error(), L


SHAPES = [((2, 2, 16, 64, 8), 80), ((3, 2, 50000, 64, 8), 64), ((1, 1, 40000, 96, 6), 1 << 20)]  # without and with a workspace
WRITTEN = dict(forward=["y", "mean", "rstd", "ws"], backward=["dx", "dgamma", "dbeta", "ws"])
OTHERS = dict(forward=["x", "gamma", "beta", "y", "mean", "rstd", "ws"],
              backward=["x", "y", "dy", "gamma", "beta", "mean", "rstd", "dx", "dgamma", "dbeta", "ws"])


@pytest.mark.parametrize("shape,par_gs", SHAPES)
@pytest.mark.parametrize("fn,out,other", [(fn, a, b) for fn in WRITTEN for a in WRITTEN[fn] for b in OTHERS[fn] if a != b])
def test_what_is_written_meets_nothing(fn, out, other, shape, par_gs):
    import paper_1808_07217_gb300 as L

    if "ws" in (out, other) and not L.lsgd_groupnorm_workspace(*shape, fn == "backward"):
        pytest.skip("no workspace at this size")
    step = 256 if "ws" in (out, other) else 4  # within the workspace's alignment
    last = lambda v: v // step * step - step  # noqa: E731
    places = [lambda a, s: a[other],  # the same address; over its first and its last bytes
              lambda a, s: a[other] - max(last(s[out]), 0), lambda a, s: a[other] + max(last(s[other]), 0)]
    for place in places:
        s, msg, L = _call(fn, shape, par_gs, **{out: place})
        assert s == L.EINVAL and "overlap" in msg, (s, msg)


@pytest.mark.parametrize("fn,out,other", [("backward", "dgamma", "dbeta"), ("backward", "dgamma", "gamma"), ("backward", "dbeta", "beta"),
                                          ("forward", "mean", "gamma"), ("forward", "y", "beta"), ("backward", "dx", "dgamma")])
@pytest.mark.parametrize("worker", [-2, -1, 1, 2])
def test_another_workers_parameters_are_met_too(fn, out, other, worker):
    """Three workers: a tensor over parameters of the second or third."""
    shape, par_gs = (3, 2, 16, 64, 8), 400
    if worker < 0 and out in ("mean", "y", "dx"):
        worker = -worker
    for edge in (lambda s: 0, lambda s: 4 - min(s[out], 256), lambda s: 252):  # the same, and a value in common at either end
        s, msg, L = _call(fn, shape, par_gs, **{out: lambda a, s: a[other] + 4 * worker * par_gs + edge(s)})
        assert s == L.EINVAL and "overlap" in msg, (s, msg)


@pytest.mark.gpu
def test_parameters_and_statistics_of_one_buffer():
    """gamma, beta, their gradients and the statistics side by side in one replica-major buffer: the same values as apart."""
    import torch

    from _gpu_common import built_package

    P = built_package()
    G, B, Pn, C, groups = 3, 2, 50, 24, 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, dy, gamma, beta = rand(G, B, Pn, C), rand(G, B, Pn, C), rand(G, C), rand(G, C)
    e = dict(device="cuda")

    def run(gamma, beta, dgamma, dbeta, mean, rstd, par_gs):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        P.lsgd_groupnorm_forward(x, gamma, beta, y, mean, rstd, G, B, Pn, C, groups, act=P.ACT_SILU, par_gs=par_gs)
        P.lsgd_groupnorm_backward(x, None, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, G, B, Pn, C, groups, act=P.ACT_SILU,
                                  par_gs=par_gs)
        torch.cuda.synchronize()
        return y, dx, mean.clone(), rstd.clone()

    dg, db = torch.empty(G, C, **e), torch.empty(G, C, **e)
    stats = [torch.empty(B * G * groups, **e) for _ in range(2)]
    want = run(gamma, beta, dg, db, *stats, C)
    d = 4 * C + 2 * B * G * groups  # gamma, beta, dgamma, dbeta, then (in the first worker's part) mean and rstd
    buf = torch.full((G, d), 77.0, **e)
    buf[:, :C], buf[:, C:2 * C] = gamma, beta
    flat = buf.view(-1)
    at = lambda k: flat[k * C:]  # noqa: E731
    ns = B * G * groups
    got = run(at(0), at(1), at(2), at(3), flat[4 * C:4 * C + ns], flat[4 * C + ns:4 * C + 2 * ns], d)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert torch.equal(buf[:, 2 * C:3 * C], dg) and torch.equal(buf[:, 3 * C:4 * C], db)
    assert torch.equal(buf[:, :C], gamma) and torch.equal(buf[:, C:2 * C], beta) and (buf[1:, 4 * C:] == 77).all()
