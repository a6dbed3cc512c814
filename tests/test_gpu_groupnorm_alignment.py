"""Group norm of tensors that start anywhere: each of them alone off its vectors' alignment, in every form."""
import pytest

import test_gpu_groupnorm as T
from _gpu_common import built_package


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


def _shifted(torch, t, k):
    """t's values k elements behind an allocation's start, a marker before and behind them."""
    n = t.numel()
    buf = torch.full((n + k + 8,), 77.0, dtype=t.dtype, device="cuda")
    buf[k:k + n] = t.reshape(-1).cuda()
    return buf, buf[k:k + n]


def _clean(buf, n, k):
    return bool((buf[:k] == 77).all()) and bool((buf[k + n:] == 77).all())


# one CTA to an image, several rounds of those with bulk copies ahead, a cluster, ranges
SHAPES = [(2, 3, 65, 64, 8), (5, 521, 64, 16, 4), (1, 4, 1517, 128, 8), (1, 1, 5000, 72, 4)]
TYPES = [("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32")]


@pytest.mark.gpu
@pytest.mark.parametrize("lead", [1, 4])
@pytest.mark.parametrize("which", ["x", "dy", "y", "dx", "all"])
@pytest.mark.parametrize("x_type,y_type", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(P, shape, x_type, y_type, which, lead):
    import torch

    G, B, Pn, C, groups = shape
    x, dy, gamma, beta, xt, yt = T._inputs(shape, C, x_type, y_type, seed=21)
    gg, bg = gamma.cuda(), beta.cuda()
    y, mean, rstd = T._run_forward(P, torch, shape, x.cuda(), gg, bg, yt, "relu", C)
    k = {name: lead if which in (name, "all") else 0 for name in ("x", "dy", "y", "dx")}
    n = x.numel()
    _, xs = _shifted(torch, x, k["x"])
    _, ds = _shifted(torch, dy, k["dy"])
    _, ys = _shifted(torch, y, k["y"])
    xbuf, dx = _shifted(torch, torch.zeros(n, dtype=xt), k["dx"])
    dgamma, dbeta = torch.empty(G, C, device="cuda"), torch.empty(G, C, device="cuda")
    P.lsgd_groupnorm_backward(xs, ys, ds, gg, bg, mean, rstd, dx, dgamma, dbeta, G, B, Pn, C, groups, act=P.ACT_RELU)
    torch.cuda.synchronize()
    assert P.lsgd_device_status() == P.OK and _clean(xbuf, n, k["dx"])
    T._check_backward(shape, x, dy, gamma, beta, y, mean, rstd, dx, dgamma, dbeta, "relu", x_type)


# the same forms; long images, whose first pass has bulk copies where x allows
@pytest.mark.gpu
@pytest.mark.parametrize("lead", [1, 4])
@pytest.mark.parametrize("which", ["x", "y", "all"])
@pytest.mark.parametrize("x_type,y_type", TYPES)
@pytest.mark.parametrize("shape", [(5, 521, 64, 16, 4), (1, 4, 1517, 128, 8), (1, 2, 13001, 168, 42)])
def test_forward(P, shape, x_type, y_type, which, lead):
    import torch

    G, B, Pn, C, groups = shape
    x, _, gamma, beta, xt, yt = T._inputs(shape, C, x_type, y_type, seed=22)
    n = x.numel()
    _, xs = _shifted(torch, x, lead if which != "y" else 0)
    ybuf, y = _shifted(torch, torch.zeros(n, dtype=yt), lead if which != "x" else 0)
    mean, rstd = torch.empty(G * B * groups, device="cuda"), torch.empty(G * B * groups, device="cuda")
    P.lsgd_groupnorm_forward(xs, gamma.cuda(), beta.cuda(), y, mean, rstd, G, B, Pn, C, groups, act=P.ACT_SILU)
    torch.cuda.synchronize()
    assert P.lsgd_device_status() == P.OK and _clean(ybuf, n, lead if which != "x" else 0)
    T._check_forward(shape, x, gamma, beta, y, mean, rstd, "silu", T.U16 if y_type == "bf16" else T.U32)
