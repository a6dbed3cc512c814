"""Group norm with an activation, forward and backward, against its definition in 64 bits."""
import ctypes

import numpy as np
import pytest

import _operator_refs as R
from _gpu_common import built_package

U32, U16 = 2.0 ** -24, 2.0 ** -8  # largest relative roundings of fp32 and bf16
ACTS = {"none": 0, "relu": 1, "silu": 2}

# (G, B, P, C, groups): single values, odd sizes, groups narrower and wider than a vector, one group and a group per
# channel, more channels than a block has threads, images of many ranges, images of one position
SHAPES = [(1, 1, 1, 1, 1), (2, 3, 5, 6, 3), (1, 2, 64, 64, 8), (2, 2, 49, 90, 9), (1, 1, 1000, 320, 32),
          (1, 2, 17, 1100, 11), (1, 1, 3, 4104, 2), (3, 2, 1, 24, 4), (2, 1, 333, 16, 16), (1, 3, 257, 40, 1),
          (1, 1, 5000, 72, 4), (2, 40, 30, 12, 2), (1, 2, 1025, 130, 10), (1, 1, 33, 2048, 1), (1, 1, 40000, 8, 1),
          (1, 2, 2000, 256, 16), (2, 1, 700, 512, 8), (1, 1, 311, 258, 6)]
# more images than the SMs hold at once: a CTA takes several, with the next ones' loads under way (and where the sizes are
# odd, one each); few and many groups, a worker's images ending between two of a CTA's
MANY = [(5, 521, 64, 16, 4), (3, 800, 9, 24, 24), (2, 1300, 100, 8, 1), (7, 90, 1024, 16, 4), (2, 611, 1, 64, 8), (1, 2500, 16, 6, 3),
        (11, 60, 260, 64, 16), (1, 3, 40000, 96, 6), (2, 1, 60001, 40, 8), (1, 12, 5003, 256, 1), (1, 2, 9001, 1536, 8),
        (2, 16, 5000, 48, 4), (4, 16, 2500, 48, 4)]


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


def _inputs(shape, par_gs, x_type, y_type, seed=0, offset=0.0):
    import torch

    G, B, Pn, C, groups = shape
    rng = np.random.default_rng(seed + sum(shape))
    t = {"bf16": torch.bfloat16, "fp32": torch.float32}
    x = torch.tensor(rng.standard_normal((G, B, Pn, C)) * 1.5 + rng.standard_normal(C) + offset, dtype=torch.float32).to(t[x_type])
    dy = torch.tensor(rng.standard_normal((G, B, Pn, C)), dtype=torch.float32).to(t[y_type])
    par = torch.tensor(np.concatenate([1 + 0.3 * rng.standard_normal((G, par_gs)), 0.3 * rng.standard_normal((G, par_gs))]),
                       dtype=torch.float32).reshape(2, G, par_gs)
    return x, dy, par[0].contiguous(), par[1].contiguous(), t[x_type], t[y_type]


def _guarded(torch, n, dtype, lead=8):
    """A tensor inside a larger one of a marker value, to see writes outside it."""
    buf = torch.full((n + 2 * lead,), 77.0, dtype=dtype, device="cuda")
    return buf, buf[lead:lead + n]


def _intact(buf, n, lead=8):
    return bool((buf[:lead] == 77).all()) and bool((buf[lead + n:] == 77).all())


def _run_forward(P, torch, shape, x, gamma, beta, yt, act, par_gs, lead=8, **kw):
    G, B, Pn, C, groups = shape
    n, ng = G * B * Pn * C, G * B * groups
    ybuf, y = _guarded(torch, n, yt, lead)
    mbuf, mean = _guarded(torch, ng, torch.float32)
    rbuf, rstd = _guarded(torch, ng, torch.float32)
    P.lsgd_groupnorm_forward(x, gamma, beta, y, mean, rstd, G, B, Pn, C, groups, act=ACTS[act], par_gs=par_gs, **kw)
    torch.cuda.synchronize()
    assert _intact(ybuf, n, lead) and _intact(mbuf, ng) and _intact(rbuf, ng)
    return y, mean, rstd


def _chain(shape):
    """Roundings that a value of a statistic passes through: a thread's run of positions (at most 64 here, four to a
    merge), the block's and the ranges' merges and the channels of a group, each a handful; 160 bounds them all."""
    return 160


def _check_forward(shape, x, gamma, beta, y, mean, rstd, act, yu, eps=1e-5):
    G, B, Pn, C, groups = shape
    xd = x.float().cpu().numpy().astype(np.float64).reshape(G, B, Pn, C)
    ga, be = (v.cpu().numpy().astype(np.float64)[:, :C] for v in (gamma, beta))
    wy, wm, wr, z = R.gn_forward(xd, ga, be, groups, eps, act)
    v = xd.reshape(G, B, Pn, groups, C // groups)
    big = np.abs(v).max((2, 4))  # a mean is off by its roundings times the largest value
    dm = _chain(shape) * U32 * big
    assert (np.abs(mean.cpu().numpy().reshape(wm.shape) - wm) <= dm).all()
    # rstd: the variance's own roundings (halved by the root), the mean's error squared, the root's rounding
    dr = wr * (_chain(shape) * U32 + (dm * wr) ** 2)
    assert (np.abs(rstd.cpu().numpy().reshape(wr.shape) - wr) <= dr).all()
    wide = lambda t: np.repeat(t[:, :, None, :], C // groups, 3)  # noqa: E731
    g = np.abs(ga)[:, None, None]
    dz = g * (wide(dm * wr) + np.abs((xd - wide(wm)) * wide(wr)) * wide(dr / wr)) + 8 * U32 * (np.abs(z) + g * (np.abs(xd) + wide(np.abs(wm))) * wide(wr) + np.abs(be)[:, None, None])
    # |act'| <= 1.1; the activation's own roundings (bf16 results take the fast exponential: 2 + |z| units, below 2^-18)
    dact = (16 * U32 if yu == U32 else 2.0 ** -18) * np.abs(wy)
    tol = 1.1 * dz + dact + yu * np.abs(wy) + 1e-37
    got = y.float().cpu().numpy().reshape(wy.shape)
    worst = np.abs(got - wy) / tol
    assert worst.max() <= 1.0, worst.max()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(P, shape, x_type, y_type, act):
    import torch

    G, B, Pn, C, groups = shape
    par_gs = C + (7 if G > 1 else 0)
    x, _, gamma, beta, xt, yt = _inputs(shape, par_gs, x_type, y_type)
    xg, gg, bg = x.cuda(), gamma.cuda(), beta.cuda()
    y, mean, rstd = _run_forward(P, torch, shape, xg, gg, bg, yt, act, par_gs)
    _check_forward(shape, x, gamma, beta, y, mean, rstd, act, U16 if y_type == "bf16" else U32)


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", ["bf16", "fp32"])
@pytest.mark.parametrize("lead", [1, 2, 4])
def test_forward_of_unaligned_tensors(P, x_type, lead):
    import torch

    shape = (2, 3, 65, 64, 8)
    G, B, Pn, C, groups = shape
    x, _, gamma, beta, xt, yt = _inputs(shape, C, x_type, x_type)
    n = x.numel()
    buf = torch.full((n + lead,), float("nan"), dtype=xt, device="cuda")
    buf[lead:] = x.reshape(-1).cuda()
    y, mean, rstd = _run_forward(P, torch, shape, buf[lead:], gamma.cuda(), beta.cuda(), yt, "silu", C, lead=lead)
    _check_forward(shape, x, gamma, beta, y, mean, rstd, "silu", U16 if x_type == "bf16" else U32)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 2, 49, 90, 9), (1, 1, 5000, 72, 4), (1, 2, 64, 64, 8)])
def test_mean_far_above_the_deviation(P, shape):
    import torch

    C = shape[3]
    x, _, gamma, beta, xt, yt = _inputs(shape, C, "fp32", "fp32", offset=3000.0)
    y, mean, rstd = _run_forward(P, torch, shape, x.cuda(), gamma.cuda(), beta.cuda(), yt, "none", C)
    _check_forward(shape, x, gamma, beta, y, mean, rstd, "none", U32)
    # a variance taken as the difference of two second moments would be off by 3000^2 2^-24 ~ 0.5 here
    xd = x.numpy().astype(np.float64)
    want = R.gn_forward(xd, gamma.numpy(), beta.numpy(), shape[4], 1e-5, "none")[2]
    assert np.abs(rstd.cpu().numpy().reshape(want.shape) / want - 1).max() < 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, 2, 64, 64, 8), (1, 1, 5000, 72, 4)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_value_that_is_not_finite_stays_in_its_group(P, shape, bad):
    import torch

    G, B, Pn, C, groups = shape
    x, _, gamma, beta, xt, yt = _inputs(shape, C, "fp32", "bf16")
    clean = _run_forward(P, torch, shape, x.cuda(), gamma.cuda(), beta.cuda(), yt, "relu", C)
    x[0, 0, Pn // 2, 3] = bad
    y, mean, rstd = _run_forward(P, torch, shape, x.cuda(), gamma.cuda(), beta.cuda(), yt, "relu", C)
    D = C // groups
    hit = torch.zeros(G, B, Pn, C, dtype=torch.bool, device="cuda")
    hit[0, 0, :, :D] = True
    hit = hit.reshape(-1)
    assert torch.isnan(y[hit].float()).all()
    assert torch.equal(y[~hit], clean[0][~hit])
    assert torch.equal(mean[1:], clean[1][1:]) and torch.equal(rstd[1:], clean[2][1:])


@pytest.mark.gpu
def test_a_group_of_equal_values(P):
    import torch

    shape = (1, 2, 64, 64, 8)
    x = torch.full((1, 2, 64, 64), 1.75, device="cuda")
    gamma, beta = torch.ones(1, 64, device="cuda"), torch.full((1, 64), 0.5, device="cuda")
    y, mean, rstd = _run_forward(P, torch, shape, x, gamma, beta, torch.float32, "none", 64)
    assert (mean == 1.75).all() and (y == 0.5).all()
    assert (rstd - 1e-5 ** -0.5).abs().max() <= 8 * U32 * 1e-5 ** -0.5


def _run_backward(P, torch, shape, x, y, dy, gamma, beta, mean, rstd, act, par_gs, **kw):
    G, B, Pn, C, groups = shape
    n, npar = G * B * Pn * C, (G - 1) * par_gs + C
    xbuf, dx = _guarded(torch, n, x.dtype)
    gbuf, dgamma = _guarded(torch, npar, torch.float32)
    bbuf, dbeta = _guarded(torch, npar, torch.float32)
    P.lsgd_groupnorm_backward(x, y, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, G, B, Pn, C, groups,
                              act=ACTS[act], par_gs=par_gs, **kw)
    torch.cuda.synchronize()
    assert _intact(xbuf, n) and _intact(gbuf, npar) and _intact(bbuf, npar)
    pick = torch.arange(G, device="cuda")[:, None] * par_gs + torch.arange(C, device="cuda")[None]
    rest = torch.ones(npar, dtype=torch.bool, device="cuda")
    rest[pick.reshape(-1)] = False
    assert (dgamma[rest] == 77).all() and (dbeta[rest] == 77).all()  # what lies between the workers' parameters
    return dx, dgamma[pick], dbeta[pick]


@pytest.mark.gpu
@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("shape", MANY)
def test_many_images(P, shape, x_type, y_type):
    import torch

    act = "silu" if (x_type == y_type) == bool(shape[0] % 2) else "relu"

    par_gs = shape[3] + 3
    x, dy, gamma, beta, xt, yt = _inputs(shape, par_gs, x_type, y_type, seed=9)
    gg, bg = gamma.cuda(), beta.cuda()
    y, mean, rstd = _run_forward(P, torch, shape, x.cuda(), gg, bg, yt, act, par_gs)
    _check_forward(shape, x, gamma, beta, y, mean, rstd, act, U16 if y_type == "bf16" else U32)
    dx, dgamma, dbeta = _run_backward(P, torch, shape, x.cuda(), y if act == "relu" else None, dy.cuda(), gg, bg, mean,
                                      rstd, act, par_gs)
    _check_backward(shape, x, dy, gamma, beta, y, mean, rstd, dx, dgamma, dbeta, act, x_type)
    assert P.lsgd_device_status() == P.OK


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(P, shape, x_type, y_type, act):
    import torch

    G, B, Pn, C, groups = shape
    par_gs = C + (7 if G > 1 else 0)
    x, dy, gamma, beta, xt, yt = _inputs(shape, par_gs, x_type, y_type, seed=5)
    gg, bg = gamma.cuda(), beta.cuda()
    y, mean, rstd = _run_forward(P, torch, shape, x.cuda(), gg, bg, yt, act, par_gs)
    dx, dgamma, dbeta = _run_backward(P, torch, shape, x.cuda(), y if act == "relu" else None, dy.cuda(), gg, bg, mean,
                                      rstd, act, par_gs)
    _check_backward(shape, x, dy, gamma, beta, y, mean, rstd, dx, dgamma, dbeta, act, x_type)


def _check_backward(shape, x, dy, gamma, beta, y, mean, rstd, dx, dgamma, dbeta, act, x_type):
    G, B, Pn, C, groups = shape
    f64 = lambda t, *s: t.float().cpu().numpy().astype(np.float64).reshape(*s)  # noqa: E731
    xd, dyd = f64(x, G, B, Pn, C), f64(dy, G, B, Pn, C)
    ga, be = f64(gamma, G, -1)[:, :C], f64(beta, G, -1)[:, :C]
    m, r = f64(mean, G, B, groups), f64(rstd, G, B, groups)
    pos = f64(y, G, B, Pn, C) > 0
    wdx, wdg, wdb, dz, xh = R.gn_backward(xd, dyd, ga, be, m, r, groups, act, pos)
    # each dz is off by its own arithmetic: 8 roundings, or SiLU's derivative (of size 1.1, its z off by 8 roundings of
    # its terms; with bf16 tensors the fast exponential's 2^-18)
    wide = lambda t: np.repeat(t[:, :, None, :], C // groups, 3)  # noqa: E731
    off = 8 * U32 * ((np.abs(xd) + wide(np.abs(m))) * wide(r))  # of xh
    ez = 8 * U32 * np.abs(dz)
    if act == "silu":
        z_off = np.abs(ga)[:, None, None] * off + 8 * U32 * (np.abs(xh * ga[:, None, None]) + np.abs(be)[:, None, None])
        ez = np.abs(dyd) * (z_off + (32 * U32 if x_type == "fp32" else 2.0 ** -18) * 1.1)
    k = _chain(shape) * U32
    tdb = ez.sum((1, 2)) + k * np.abs(dz).sum((1, 2))
    tdg = (ez * np.abs(xh) + np.abs(dz) * off).sum((1, 2)) + k * np.abs(dz * xh).sum((1, 2))
    got = lambda t: t.cpu().numpy().reshape(G, C)  # noqa: E731
    assert (np.abs(got(dbeta) - wdb) <= tdb + 1e-37).all()
    assert (np.abs(got(dgamma) - wdg) <= tdg + 1e-37).all()
    s = (G, B, Pn, groups, C // groups)
    g = np.abs(ga)[:, None, None]
    mean_of = lambda t: t.reshape(s).mean((2, 4))  # noqa: E731
    e1 = mean_of(g * ez + k * g * np.abs(dz))
    e2 = mean_of(g * (ez * np.abs(xh) + np.abs(dz) * off) + k * g * np.abs(dz * xh))
    m2 = wide(mean_of(ga[:, None, None] * dz * xh))
    tol = wide(r) * (g * ez + wide(e1) + np.abs(xh) * wide(e2) + off * np.abs(m2) +
                     8 * U32 * (g * np.abs(dz) + wide(mean_of(g * np.abs(dz))) + np.abs(xh) * np.abs(m2)))
    tol = tol + (U16 if x_type == "bf16" else U32) * np.abs(wdx) + 1e-37
    worst = np.abs(f64(dx, G, B, Pn, C) - wdx) / tol
    assert worst.max() <= 1.0, worst.max()


# images that clusters of nine and of ten CTAs hold, in one of the directions or both, and one image more than run at once
@pytest.mark.gpu
@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("shape", [(3, 5, 1517, 90, 9), (3, 3, 1517, 90, 9), (2, 5, 3001, 90, 9), (1, 13, 1040, 128, 16),
                                   (2, 8, 1517, 90, 9), (1, 9, 2401, 64, 1), (1, 15, 130, 1024, 32)])
def test_clusters_of_nine_and_ten(P, shape, x_type, y_type):
    import torch

    par_gs = shape[3] + 2
    x, dy, gamma, beta, xt, yt = _inputs(shape, par_gs, x_type, y_type, seed=13)
    gg, bg = gamma.cuda(), beta.cuda()
    y, mean, rstd = _run_forward(P, torch, shape, x.cuda(), gg, bg, yt, "relu", par_gs)
    _check_forward(shape, x, gamma, beta, y, mean, rstd, "relu", U16 if y_type == "bf16" else U32)
    dx, dgamma, dbeta = _run_backward(P, torch, shape, x.cuda(), y, dy.cuda(), gg, bg, mean, rstd, "relu", par_gs)
    _check_backward(shape, x, dy, gamma, beta, y, mean, rstd, dx, dgamma, dbeta, "relu", x_type)


# images that no cluster holds: ranges of a few positions and of many; one group, groups within and across vectors; one
# position's channels wider than the threads; many images
LARGE = [(1, 1, 60007, 24, 1), (1, 2, 13001, 168, 42), (2, 3, 20011, 104, 13), (1, 1, 701, 2048, 64), (1, 1, 301, 4096, 2),
         (2, 88, 1101, 480, 4), (2, 4, 940, 484, 2), (1, 3, 2000, 500, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("fp32", "bf16")])
@pytest.mark.parametrize("shape", LARGE)
def test_forward_of_large_images(P, shape, x_type, y_type):
    import torch

    if shape[0] * shape[1] > 100 and x_type == "fp32":
        pytest.skip("the same path as bf16, twice the oracle's time")
    par_gs = shape[3] + 1
    x, _, gamma, beta, xt, yt = _inputs(shape, par_gs, x_type, y_type, seed=3)
    y, mean, rstd = _run_forward(P, torch, shape, x.cuda(), gamma.cuda(), beta.cuda(), yt, "silu", par_gs)
    _check_forward(shape, x, gamma, beta, y, mean, rstd, "silu", U16)
    assert P.lsgd_device_status() == P.OK


@pytest.mark.gpu
def test_large_images_twice_at_once_captured_and_with_values_that_are_not_finite(P):
    import torch

    shape = G, B, Pn, C, groups = (1, 2, 13001, 168, 42)
    x, _, gamma, beta, xt, yt = _inputs(shape, C, "bf16", "bf16")
    clean = _run_forward(P, torch, shape, x.cuda(), gamma.cuda(), beta.cuda(), yt, "relu", C)
    # a NaN in one image's group reaches the image's CTAs and no other group
    x[0, 1, Pn // 3, 9] = float("nan")
    xg, gg, bg, e = x.cuda(), gamma.cuda(), beta.cuda(), dict(device="cuda")
    y, mean, rstd = _run_forward(P, torch, shape, xg, gg, bg, yt, "relu", C)
    hit = torch.zeros(G, B, Pn, C, dtype=torch.bool, device="cuda")
    hit[0, 1, :, 8:12] = True
    hit = hit.reshape(-1)
    assert torch.isnan(y[hit].float()).all() and torch.equal(y[~hit], clean[0][~hit])
    # two streams' calls at once, a graph replayed, workspaces full of anything: the same bits
    need = P.lsgd_groupnorm_workspace(G, B, Pn, C, groups, False)
    outs = [(torch.empty_like(xg), torch.empty(B * groups, **e), torch.empty(B * groups, **e),
             torch.full((need,), 255 * (i % 2), dtype=torch.uint8, **e)) for i in range(3)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()

    def call(o, **kw):
        P.lsgd_groupnorm_forward(xg, gg, bg, o[0], o[1], o[2], G, B, Pn, C, groups, act=P.ACT_RELU, workspace=o[3], **kw)

    for _ in range(5):
        for st, o in zip(streams, outs):
            call(o, stream=st.cuda_stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[2])
    for _ in range(3):
        outs[2][3].random_()
        graph.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[0].reshape(-1).view(torch.int16), y.view(torch.int16))
        assert torch.equal(o[1].view(torch.int32), mean.view(torch.int32))
        assert torch.equal(o[2].view(torch.int32), rstd.view(torch.int32))
    assert P.lsgd_device_status() == P.OK


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 3, 65, 64, 8), (1, 1, 5000, 72, 4), (2, 2, 49, 90, 9)])
def test_same_bits_every_time_captured_and_on_another_stream(P, shape):
    import torch

    G, B, Pn, C, groups = shape
    x, dy, gamma, beta, xt, yt = _inputs(shape, C, "bf16", "bf16")
    x, dy, gamma, beta = x.cuda(), dy.cuda(), gamma.cuda(), beta.cuda()
    e = dict(device="cuda")

    def buffers():
        return dict(y=torch.empty_like(x), mean=torch.empty(G * B * groups, **e), rstd=torch.empty(G * B * groups, **e),
                    dx=torch.empty_like(x), dgamma=torch.empty(G, C, **e), dbeta=torch.empty(G, C, **e))

    def both(b, **kw):
        P.lsgd_groupnorm_forward(x, gamma, beta, b["y"], b["mean"], b["rstd"], G, B, Pn, C, groups, act=P.ACT_SILU, **kw)
        P.lsgd_groupnorm_backward(x, None, dy, gamma, beta, b["mean"], b["rstd"], b["dx"], b["dgamma"], b["dbeta"], G,
                                  B, Pn, C, groups, act=P.ACT_SILU, **kw)

    want = buffers()
    both(want)
    torch.cuda.synchronize()
    again = buffers()
    both(again)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other, named, played = buffers(), buffers(), buffers()
    with torch.cuda.stream(side):
        both(other)
    both(named, stream=side.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(played)
    for _ in range(2):
        for v in played.values():
            v.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        for got in (again, other, named, played):
            for k in want:
                assert torch.equal(got[k], want[k]), k


# ------------------------------------------------------------------ refusals, without a GPU


def _call(fn, **kw):
    """The C call with plausible arguments (addresses that are never used: every call here is refused)."""
    from paper_1808_07217_gb300 import _build

    _build.build()
    import paper_1808_07217_gb300 as L

    base = dict(x=1 << 20, x_type=1, gamma=2 << 20, beta=3 << 20, par_gs=64, y=4 << 20, y_type=1, mean=5 << 20, rstd=6 << 20,
                dy=7 << 20, dx=8 << 20, dgamma=9 << 20, dbeta=10 << 20, G=2, B=2, P=16, C=64, groups=8, eps=1e-5, act=1,
                ws=11 << 20, wn=1 << 20)
    base.update(kw)
    a = base
    vp = lambda k: ctypes.c_void_p(a[k])  # noqa: E731
    if fn == "forward":
        s = L.lib().lsgd_groupnorm_forward(vp("x"), a["x_type"], vp("gamma"), vp("beta"), a["par_gs"], vp("y"),
                                           a["y_type"], vp("mean"), vp("rstd"), a["G"], a["B"], a["P"], a["C"],
                                           a["groups"], a["eps"], a["act"], vp("ws"), a["wn"], None)
    else:
        s = L.lib().lsgd_groupnorm_backward(vp("x"), a["x_type"], vp("y"), vp("dy"), a["y_type"], vp("gamma"),
                                            vp("beta"), a["par_gs"], vp("mean"), vp("rstd"), vp("dx"), vp("dgamma"),
                                            vp("dbeta"), a["G"], a["B"], a["P"], a["C"], a["groups"], a["act"],
                                            vp("ws"), a["wn"], None)
    return s, L.lsgd_last_error(), L.EINVAL


_BOTH = [dict(G=0), dict(B=0), dict(P=0), dict(C=0), dict(groups=0), dict(groups=7), dict(groups=-8), dict(x=None),
         dict(gamma=None), dict(beta=None), dict(mean=None), dict(rstd=None), dict(x_type=2), dict(y_type=-1), dict(act=3),
         dict(act=-1), dict(par_gs=63), dict(ws=None, P=50000), dict(wn=15, P=50000), dict(ws=(11 << 20) + 8, P=50000), dict(x=(1 << 20) + 1),
         dict(gamma=(2 << 20) + 2), dict(G=70000), dict(G=5000, B=5000), dict(P=(1 << 24) + 1), dict(C=65544),
         dict(ws=(1 << 20) + 64)]


@pytest.mark.parametrize("kw", _BOTH + [dict(y=None), dict(y=1 << 20), dict(y=(1 << 20) + 16), dict(eps=0.0),
                                        dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(mean=6 << 20),
                                        dict(y=(4 << 20) + 1)])
def test_forward_refuses(kw):
    s, msg, want = _call("forward", **kw)
    assert s == want and msg.startswith("lsgd_groupnorm_forward: "), (s, msg)


@pytest.mark.parametrize("kw", _BOTH + [dict(y=None), dict(dy=None), dict(dx=None), dict(dgamma=None), dict(dbeta=None),
                                        dict(dx=1 << 20), dict(dx=7 << 20), dict(dx=4 << 20), dict(dgamma=10 << 20),
                                        dict(dy=(7 << 20) + 1), dict(dgamma=(9 << 20) + 2), dict(y=(4 << 20) + 1)])
def test_backward_refuses(kw):
    s, msg, want = _call("backward", **kw)
    assert s == want and msg.startswith("lsgd_groupnorm_backward: "), (s, msg)


def test_workspace_refuses_and_grows():
    from paper_1808_07217_gb300 import _build

    _build.build()
    import paper_1808_07217_gb300 as L

    for bad in ((0, 1, 1, 1, 1), (1, 1, 1, 6, 4), (1, 1, 0, 6, 3)):
        with pytest.raises(L.LsgdError) as e:
            L.lsgd_groupnorm_workspace(*bad)
        assert e.value.status == L.EINVAL
    for P in (64, 100000):  # few positions stay in registers, many are split over ranges
        assert (L.lsgd_groupnorm_workspace(2, 2, P, 64, 8) > 0) == (P > 64)
        assert L.lsgd_groupnorm_workspace(2, 2, P, 64, 8) < L.lsgd_groupnorm_workspace(2, 2, P, 64, 8, backward=True)


def test_binding_refuses_host_and_short_tensors():
    import torch

    from paper_1808_07217_gb300 import _build

    _build.build()
    import paper_1808_07217_gb300 as L

    t = torch.zeros(2, 2, 16, 64)
    s = torch.zeros(2, 2, 8)
    with pytest.raises(L.LsgdError) as e:
        L.lsgd_groupnorm_forward(t, torch.ones(2, 64), torch.ones(2, 64), t.clone(), s, s.clone(), 2, 2, 16, 64, 8)
    assert e.value.status == L.EINVAL


@pytest.mark.gpu
def test_binding_refuses_wrong_tensors(P):
    import torch

    G, B, Pn, C, groups = 2, 2, 16, 64, 8
    e = dict(device="cuda")
    ok = dict(x=torch.zeros(G, B, Pn, C, **e), gamma=torch.ones(G, C, **e), beta=torch.ones(G, C, **e),
              y=torch.zeros(G, B, Pn, C, **e), mean=torch.zeros(G, B, groups, **e), rstd=torch.zeros(G, B, groups, **e))
    for bad in (dict(x=ok["x"].half()), dict(x=ok["x"].transpose(2, 3)), dict(y=ok["y"][:, :1].contiguous()),
                dict(mean=ok["mean"].double()), dict(gamma=ok["gamma"][:1].contiguous()), dict(beta=ok["beta"].cpu()),
                dict(gamma=ok["gamma"].bfloat16())):
        with pytest.raises(P.LsgdError) as err:
            P.lsgd_groupnorm_forward(*{**ok, **bad}.values(), G, B, Pn, C, groups)
        assert err.value.status == P.EINVAL
    with pytest.raises(P.LsgdError) as err:
        P.lsgd_groupnorm_backward(ok["x"], None, ok["y"], ok["gamma"], ok["beta"], ok["mean"], ok["rstd"], ok["x"].clone(),
                                  ok["gamma"].clone(), ok["beta"].clone(), G, B, Pn, C, groups, workspace=torch.zeros(16, **e))
    assert err.value.status == P.EINVAL
