"""Orthogonalised update directions and their application, against the definitions in 64 bits."""

import numpy as np
import pytest

import _operator_refs as R
from _gpu_common import built_package

U32, U16 = 2.0 ** -24, 2.0 ** -8
# How far a direction may be off before its bf16 rounding, of its 2-norm.  A step rounds A and P (and above a smaller side of
# 64 X as an operand) to fp16, 2^-11 of each value at most and 2^-11 / sqrt(3) = 2.8e-4 in the mean; |P| < 2.9, so a step's
# rounding of P alone moves X by up to 8e-4, and the steps after it multiply what lies in X's space by a slope that is
# below one near the plateau: the last two or three steps count, 1.5e-3 in all.  Matrices of a few values do not average:
# CPU models of the same roundings gave at most 2.4e-3 over thousands of tiny and degenerate ones.
def _off(shape):
    return 2.5e-3 if min(shape[1:]) <= 64 else 1.5e-3


# (G, rows, cols): single values, vectors, odd sizes, both orientations, sizes on, below and above every tile (64, 128,
# 256), more matrices than CTA pairs, a long row
SHAPES = [(1, 1, 1), (3, 1, 7), (2, 7, 1), (4, 16, 144), (2, 10, 1024), (3, 64, 576), (2, 576, 64), (1, 100, 4096),
          (1, 130, 131), (1, 131, 130), (2, 128, 128), (1, 129, 300), (2, 256, 256), (1, 257, 257), (1, 300, 1031),
          (1, 1031, 300), (1, 512, 700), (160, 20, 36), (1, 24, 9000), (2, 9000, 24), (1, 1, 5000), (1, 640, 640),
          (2, 127, 127), (1, 255, 900), (1, 100, 5000), (1, 2049, 130), (21, 70, 2100), (17, 2300, 30), (40, 12, 4096), (3, 128, 20000), (2, 100, 700), (1, 24, 2100), (3, 5100, 90), (1, 300, 40), (20, 33, 900)]


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


def _matrix(rng, shape, kind):
    G, rows, cols = shape
    if kind == "random":
        return rng.standard_normal(shape)
    if kind == "low_rank":  # a gradient of a mini-batch smaller than the layer
        r = max(1, min(rows, cols) // 16)
        return rng.standard_normal((G, rows, r)) @ rng.standard_normal((G, r, cols)) / r
    if kind == "graded":  # columns of very different sizes
        return rng.standard_normal(shape) * np.exp(2 * rng.standard_normal((G, 1, cols)))
    raise ValueError(kind)


def _guarded(torch, n, dtype, lead=16):
    buf = torch.full((n + 2 * lead,), 77.0, dtype=dtype, device="cuda")
    return buf, buf[lead:lead + n]


def _run(P, torch, shape, u, g, momentum=0.95, nesterov=True, steps=5, gs=0, lead=16, **kw):
    """u and g [G][rows * cols] arrays; returns u and o [G][rows][cols] as computed.  gs: extra elements between matrices."""
    G, rows, cols = shape
    n = rows * cols
    stride = n + gs
    span = (G - 1) * stride + n

    def spread(src, dtype):
        buf, t = _guarded(torch, span, dtype, lead)
        for k in range(G):
            t[k * stride:k * stride + n] = src[k].reshape(-1)
        return buf, t

    gbuf, gt = spread(g, g.dtype)
    obuf, ot = _guarded(torch, span, torch.bfloat16, lead)
    ubuf, ut = spread(u, torch.float32) if u is not None else (None, None)
    P.lsgd_orthogonal_direction(ut, gt, ot, G, rows, cols, momentum=momentum, nesterov=nesterov, steps=steps, u_gs=stride,
                                g_gs=stride, o_gs=stride, **kw)
    torch.cuda.synchronize()
    assert P.lsgd_device_status() == P.OK
    keep = torch.zeros(span + 2 * lead, dtype=torch.bool, device="cuda")
    for k in range(G):
        keep[lead + k * stride:lead + k * stride + n] = True
    for buf in (gbuf, obuf, ubuf):
        if buf is not None:
            assert (buf[~keep] == 77).all()  # nothing outside the matrices is written
    pick = lambda t: torch.stack([t[k * stride:k * stride + n] for k in range(G)]).reshape(shape)  # noqa: E731
    return pick(ut) if ut is not None else None, pick(ot)


def _check(o, x, steps=5):
    """o against the definition for x (64 bits): what it may be off, and its rounding to bf16 (that of the exact values where
    they are many, which is the same to a tenth; at most 2^-8 of each otherwise)."""
    import torch

    want = R.direction(x, steps)
    got = o.float().cpu().numpy().astype(np.float64)
    for k in range(len(want)):
        norm = np.linalg.norm(want[k])
        off = np.linalg.norm(got[k] - want[k])
        rounded = np.linalg.norm(torch.tensor(want[k]).bfloat16().double().numpy() - want[k])
        rounding = 1.1 * rounded if want[k].size >= 256 else U16 * norm
        assert off <= norm * _off(x.shape) + rounding and np.isfinite(got[k]).all(), (k, off / norm)
        # no single value is far off either: the error is spread over the matrix, not in one tile
        rms, big = norm / np.sqrt(want[k].size), np.abs(want[k]).max()
        assert np.abs(got[k] - want[k]).max() <= U16 * big + 1e-2 * 8 * max(rms, big / 8)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["random", "low_rank", "graded"])
@pytest.mark.parametrize("shape", SHAPES)
def test_direction(P, shape, kind):
    import torch

    G, rows, cols = shape
    rng = np.random.default_rng(G + 7 * rows + 31 * cols)
    g = torch.tensor(_matrix(rng, shape, kind) * 1e-3, dtype=torch.float32)
    u = torch.tensor(_matrix(rng, shape, kind) * 1e-2, dtype=torch.float32)
    got_u, o = _run(P, torch, shape, u.cuda(), g.cuda())
    m = np.float64(np.float32(0.95))
    want_u = m * u.double().numpy() + g.double().numpy()
    assert (np.abs(got_u.cpu().numpy() - want_u) <= U32 * np.abs(want_u) + 1e-40).all()  # one rounding (fused)
    _check(o, g.double().numpy() + m * got_u.double().cpu().numpy())


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(3, 64, 576), (2, 131, 130), (1, 300, 1031), (2, 10, 33)])
@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("momentum,nesterov", [(0.0, True), (0.0, False), (0.9, False), (0.9, True)])
def test_momentum_forms_gradient_types_and_strides(P, shape, grad, momentum, nesterov):
    import torch

    rng = np.random.default_rng(sum(shape))
    g = torch.tensor(rng.standard_normal(shape), dtype=torch.float32)
    g = g.bfloat16() if grad == "bf16" else g
    u = torch.tensor(rng.standard_normal(shape), dtype=torch.float32)
    m = np.float64(np.float32(momentum))
    for gs in (0, 13, 64):
        got_u, o = _run(P, torch, shape, u.cuda(), g.cuda(), momentum, nesterov, gs=gs, lead=16 if gs != 13 else 3)
        gd, ud = g.double().numpy(), u.double().numpy()
        if momentum == 0:
            assert torch.equal(got_u.cpu(), u)
            x = gd
        else:
            want = m * ud + gd
            assert (np.abs(got_u.cpu().numpy() - want) <= U32 * np.abs(want) + 1e-40).all()
            x = got_u.double().cpu().numpy()
            x = gd + m * x if nesterov else x
        _check(o, x)
    if momentum == 0:  # and without a momentum buffer at all
        _check(_run(P, torch, shape, None, g.cuda(), 0.0)[1], g.double().numpy())


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [1, 2, 3, 6])
@pytest.mark.parametrize("shape", [(2, 64, 200), (1, 300, 150)])
def test_number_of_steps(P, shape, steps):
    import torch

    g = torch.tensor(np.random.default_rng(steps).standard_normal(shape), dtype=torch.float32)
    _check(_run(P, torch, shape, None, g.cuda(), 0.0, steps=steps)[1], g.double().numpy(), steps)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(3, 40, 70), (3, 200, 170)])
@pytest.mark.parametrize("size", [1e-42, 1e-30, 1e-12, 1e12, 1e19, 1e33])
def test_matrices_of_any_size(P, shape, size):
    import torch

    x = np.random.default_rng(1).standard_normal(shape) * size
    g = torch.tensor(x, dtype=torch.float32)
    _check(_run(P, torch, shape, None, g.cuda(), 0.0)[1], g.double().numpy())


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(4, 40, 70), (4, 200, 170), (4, 170, 300)])
def test_zero_and_not_finite_matrices_keep_to_themselves(P, shape):
    import torch

    g = torch.tensor(np.random.default_rng(2).standard_normal(shape), dtype=torch.float32)
    clean = _run(P, torch, shape, None, g.cuda(), 0.0)[1]
    g[0] = 0
    g[1, 3, 5] = float("nan")
    g[2, 1, 2] = float("inf")
    o = _run(P, torch, shape, None, g.cuda(), 0.0)[1]
    assert not o[0].any()
    assert torch.isnan(o[1]).all() and torch.isnan(o[2]).all()
    assert torch.equal(o[3], clean[3])


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(3, 64, 576), (2, 300, 257), (3, 40, 5000), (1, 4600, 100)])
def test_same_bits_every_time_captured_and_on_another_stream(P, shape):
    import torch

    G, rows, cols = shape
    gen = torch.Generator(device="cuda").manual_seed(4)
    g = torch.randn(shape, generator=gen, device="cuda")
    u0 = torch.randn(shape, generator=gen, device="cuda")
    w0 = torch.randn(shape, generator=gen, device="cuda")

    def step(u, w, o, wb, **kw):
        P.lsgd_orthogonal_direction(u, g, o, G, rows, cols, **kw)
        P.lsgd_direction_update(w, o, wb, G, rows * cols, 0.02, scale=1.5, weight_decay=0.1, **kw)

    def fresh():
        return u0.clone(), w0.clone(), torch.empty(shape, dtype=torch.bfloat16, device="cuda"), torch.empty(shape, dtype=torch.bfloat16, device="cuda")

    want = fresh()
    for _ in range(2):
        step(*want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other, named, played = fresh(), fresh(), fresh()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(2):
            step(*other)
    for _ in range(2):
        step(*named, stream=side.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*played)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for got in (other, named, played):
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_calls_of_every_form_at_once(P):
    """Clusters, groups that meet in global memory and both kinds of tiles on two streams, each call with its own workspace."""
    import torch

    shapes = [(20, 64, 576), (2, 40, 5000), (2, 300, 257), (1, 4600, 100), (4, 1024, 1024), (1, 300, 600)]
    gen = torch.Generator(device="cuda").manual_seed(6)
    gs = [torch.randn(s, generator=gen, device="cuda") for s in shapes]
    streams = [torch.cuda.Stream() for _ in range(2)]

    def buffers():
        return [(torch.zeros_like(g), torch.empty_like(g, dtype=torch.bfloat16),
                 torch.empty(max(P.lsgd_orthogonal_workspace(*g.shape), 1), dtype=torch.uint8, device="cuda")) for g in gs]

    def call(g, b, **kw):
        P.lsgd_orthogonal_direction(b[0], g, b[1], *g.shape, workspace=b[2], **kw)

    want = buffers()
    for _ in range(3):
        for g, b in zip(gs, want):
            call(g, b)
    got = [buffers(), buffers()]
    torch.cuda.synchronize()
    for _ in range(3):  # one stream's calls in the other order, so that different forms meet
        for i in range(len(gs)):
            call(gs[i], got[0][i], stream=streams[0].cuda_stream)
            call(gs[-1 - i], got[1][-1 - i], stream=streams[1].cuda_stream)
    torch.cuda.synchronize()
    assert P.lsgd_device_status() == P.OK
    for bs in got:
        for b, w in zip(bs, want):
            assert torch.equal(b[0], w[0]) and torch.equal(b[1], w[1])


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, 40, 72), (1, 192, 256)])
@pytest.mark.parametrize("stride", [0, 1, -8, 1 << 60])
def test_a_single_matrix_has_no_strides(P, shape, stride):
    import ctypes

    import torch

    _, rows, cols = shape
    x = np.random.default_rng(4).standard_normal(shape)
    g = torch.tensor(x, dtype=torch.float32, device="cuda")
    o = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    need = P.lsgd_orthogonal_workspace(1, rows, cols)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    st = P.lib().lsgd_orthogonal_direction(None, stride, g.data_ptr(), P.FP32, stride, o.data_ptr(), stride, 1, rows, cols,
                                           ctypes.c_float(0.0), 0, 5, ws.data_ptr(), need, None)
    torch.cuda.synchronize()
    assert st == P.OK
    _check(o, x)


@pytest.mark.gpu
@pytest.mark.parametrize("G,n,gs,lead", [(1, 1, 0, 16), (3, 17, 0, 16), (2, 4096, 0, 16), (2, 4096, 8, 8), (4, 1000, 5, 3), (1, 999, 0, 1),
                                         (64, 640, 64, 16), (2, 300001, 0, 16), (1, 1 << 20, 0, 16), (7, 4099, 0, 16),
                                         (3, 1001, 7, 16), (5, 300007, 1, 16), (1, 9, 0, 16)])
@pytest.mark.parametrize("shadow", [True, False])
def test_update(P, G, n, gs, lead, shadow):
    import torch

    rng = np.random.default_rng(n)
    stride = n + gs
    span = (G - 1) * stride + n
    wbuf, w = _guarded(torch, span, torch.float32, lead)
    obuf, o = _guarded(torch, span, torch.bfloat16, lead)
    bbuf, wb = _guarded(torch, span, torch.bfloat16, lead)
    w0 = torch.tensor(rng.standard_normal((G, n)), dtype=torch.float32)
    o0 = torch.tensor(rng.standard_normal((G, n)), dtype=torch.float32).bfloat16()
    keep = torch.zeros(span + 2 * lead, dtype=torch.bool, device="cuda")
    for k in range(G):
        w[k * stride:k * stride + n] = w0[k].cuda()
        o[k * stride:k * stride + n] = o0[k].cuda()
        keep[lead + k * stride:lead + k * stride + n] = True
    P.lsgd_direction_update(w, o, wb if shadow else None, G, n, 0.3, scale=0.7, weight_decay=0.1, w_gs=stride, o_gs=stride)
    torch.cuda.synchronize()
    for buf in (wbuf, obuf, bbuf):
        assert (buf[~keep] == 77).all()
    lr, sc, wd = (np.float64(np.float32(v)) for v in (0.3, 0.7, 0.1))
    want = (1 - lr * wd) * w0.double().numpy() - lr * sc * o0.double().numpy()
    # the two factors, the decayed weight and the sum are rounded once each
    tol = U32 * (2 * np.abs(w0.numpy()) + lr * sc * np.abs(o0.float().numpy()) + np.abs(want)) * 1.01
    got = torch.stack([w[k * stride:k * stride + n] for k in range(G)])
    assert (np.abs(got.cpu().numpy() - want) <= tol).all()
    gb = torch.stack([wb[k * stride:k * stride + n] for k in range(G)])
    assert torch.equal(gb, got.bfloat16()) if shadow else (gb == 77).all()


@pytest.mark.gpu
def test_a_layer_inside_a_replica_major_buffer(P):
    """Several steps on one layer of K replicas that stand in larger buffers, with the average after them, as a user of the
    replica-major buffers runs them."""
    import torch

    K, rows, cols, before, after = 4, 72, 96, 64, 128
    d = before + rows * cols + after
    gen = torch.Generator(device="cuda").manual_seed(8)
    W, U = torch.randn(K, d, generator=gen, device="cuda"), torch.zeros(K, d, device="cuda")
    Wb, O = torch.zeros(K, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(K, rows * cols, dtype=torch.bfloat16, device="cuda")
    W0 = W.clone()
    w, u = W.double().cpu().numpy()[:, before:before + rows * cols], np.zeros((K, rows * cols))
    m, lr, wd = (np.float64(np.float32(v)) for v in (0.95, 0.02, 0.01))
    flat = lambda t: t.view(-1)[before:]  # noqa: E731
    for s in range(3):
        Gr = torch.randn(K, d, generator=gen, device="cuda")
        P.lsgd_orthogonal_direction(flat(U), flat(Gr), O, K, rows, cols, u_gs=d, g_gs=d)
        P.lsgd_direction_update(flat(W), O, flat(Wb), K, rows * cols, 0.02, weight_decay=0.01, w_gs=d)
        gr = Gr.double().cpu().numpy()[:, before:before + rows * cols]
        u = m * u + gr
        w = (1 - lr * wd) * w - lr * R.direction((gr + m * u).reshape(K, rows, cols), 5).reshape(K, -1)
    torch.cuda.synchronize()
    got = W.double().cpu().numpy()
    # three directions of at most 1.21 in every singular value, each off by 1.5e-3 + 2^-8 of its norm, times lr
    tol = 3 * lr * (1.5e-3 + 2.0 ** -8) * 1.21 * np.sqrt(rows) + 8 * U32 * np.linalg.norm(w[0])
    for k in range(K):
        assert np.linalg.norm(got[k, before:before + rows * cols] - w[k]) <= tol
    assert torch.equal(W[:, :before], W0[:, :before]) and torch.equal(W[:, before + rows * cols:], W0[:, before + rows * cols:])
    P.lsgd_kway_average(W, Wb, K, d)
    torch.cuda.synchronize()
    assert np.abs(W[2].double().cpu().numpy() - got.mean(0)).max() <= 1e-6 * np.abs(got).mean(0).max()


# ------------------------------------------------------------------ refusals, without a GPU


def _lib():
    from paper_1808_07217_gb300 import _build

    _build.build()
    import paper_1808_07217_gb300 as L

    return L


_LARGE = dict(rows=200, cols=300, u_gs=60000, g_gs=60000, o_gs=60000)  # sizes that use a workspace
_BAD = [dict(G=0), dict(rows=0), dict(cols=0), dict(G=70000), dict(rows=32769), dict(cols=40000), dict(g=None), dict(o=None), dict(u=None),
        dict(g_type=2), dict(momentum=-0.1), dict(momentum=float("nan")), dict(momentum=float("inf")), dict(steps=0), dict(steps=101),
        dict(u_gs=10), dict(g_gs=10), dict(o_gs=10), dict(u_gs=-1 << 20), dict(u=(1 << 30) + 2), dict(g=(2 << 30) + 1), dict(o=(3 << 30) + 1),
        dict(ws=None, **_LARGE), dict(wn=100, **_LARGE), dict(ws=(4 << 30) + 16, **_LARGE), dict(o=2 << 30), dict(u=2 << 30), dict(u=3 << 30), dict(ws=1 << 30, **_LARGE),
        dict(ws=2 << 30, **_LARGE), dict(ws=3 << 30, **_LARGE)]


@pytest.mark.parametrize("kw", _BAD)
def test_direction_refuses(kw):
    L = _lib()
    a = dict(u=1 << 30, u_gs=6400, g=2 << 30, g_type=0, g_gs=6400, o=3 << 30, o_gs=6400, G=2, rows=64, cols=100, momentum=0.9,
             nesterov=1, steps=5, ws=4 << 30, wn=1 << 28)
    a.update(kw)
    assert L.lib().lsgd_orthogonal_direction(a["u"], a["u_gs"], a["g"], a["g_type"], a["g_gs"], a["o"], a["o_gs"], a["G"], a["rows"],
                                             a["cols"], a["momentum"], a["nesterov"], a["steps"], a["ws"], a["wn"], None) == L.EINVAL
    assert L.lsgd_last_error().startswith("lsgd_orthogonal_direction: ")


@pytest.mark.parametrize("kw", [dict(G=0), dict(G=70000), dict(n=0), dict(n=1 << 31), dict(w=None), dict(o=None), dict(w_gs=63), dict(o_gs=63),
                                dict(w=(1 << 30) + 2), dict(o=(2 << 30) + 1), dict(wb=(3 << 30) + 1), dict(o=1 << 30), dict(wb=1 << 30), dict(wb=2 << 30)])
def test_update_refuses(kw):
    L = _lib()
    a = dict(w=1 << 30, w_gs=64, o=2 << 30, o_gs=64, wb=3 << 30, G=2, n=64)
    a.update(kw)
    assert L.lib().lsgd_direction_update(a["w"], a["w_gs"], a["o"], a["o_gs"], a["wb"], a["G"], a["n"], 0.1, 1.0, 0.0, None) == L.EINVAL
    assert L.lsgd_last_error().startswith("lsgd_direction_update: ")


def test_workspace_refuses_and_grows():
    L = _lib()
    for bad in ((0, 4, 4), (1, 0, 4), (1, 4, 32769)):
        with pytest.raises(L.LsgdError) as e:
            L.lsgd_orthogonal_workspace(*bad)
        assert e.value.status == L.EINVAL
    assert L.lsgd_orthogonal_workspace(9, 4096, 128) == 0 < L.lsgd_orthogonal_workspace(16, 4096, 128)
    assert 0 < L.lsgd_orthogonal_workspace(1, 300, 300) < L.lsgd_orthogonal_workspace(2, 300, 300)


@pytest.mark.gpu
def test_binding_refuses_wrong_tensors(P):
    import torch

    e = dict(device="cuda")
    u, g, o = torch.zeros(2, 8, 16, **e), torch.zeros(2, 8, 16, **e), torch.zeros(2, 8, 16, dtype=torch.bfloat16, **e)
    for bad in ((u.double(), g, o), (u, g.half(), o), (u, g, o.float()), (u[:1].contiguous(), g, o), (u, g.transpose(1, 2), o),
                (u.cpu(), g, o), (None, g, o)):
        with pytest.raises(P.LsgdError) as err:
            P.lsgd_orthogonal_direction(*bad, 2, 8, 16)
        assert err.value.status == P.EINVAL
    for bad in ((u, o, o[:1].contiguous()), (u.bfloat16(), o, None), (u, u, None)):
        with pytest.raises(P.LsgdError) as err:
            P.lsgd_direction_update(*bad, 2, 128, 0.1)
        assert err.value.status == P.EINVAL
