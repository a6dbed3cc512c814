"""Group norm's sums where they are long: equal values, whose roundings all go one way, added up in 64 bits beside the kernels'
sums.  A tolerance counts the additions that a value passes through, of half a unit (2^-24) each."""
import numpy as np
import pytest

from _gpu_common import built_package

U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


def _backward(P, shape, x_type, additions, seed=0):
    """dy = 0.1 everywhere, no activation.  dx, dgamma and dbeta against 64 bits on the GPU, one worker at a time."""
    import torch

    G, B, Pn, C, groups = shape
    D = C // groups
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(G, B, Pn, C, generator=gen, device="cuda").to(x_type)
    gamma = 1 + 0.2 * torch.rand(G, C, generator=gen, device="cuda")
    beta = torch.zeros(G, C, device="cuda")
    dy = torch.full((G, B, Pn, C), 0.1, device="cuda")
    v = x.view(G, B, Pn, groups, D)
    mean = torch.stack([v[k].double().mean((1, 3)) for k in range(G)]).float()
    rstd = torch.stack([(v[k].double().var((1, 3), correction=0) + 1e-5).rsqrt() for k in range(G)]).float()
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
    P.lsgd_groupnorm_backward(x, None, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, G, B, Pn, C, groups)
    torch.cuda.synchronize()
    assert P.lsgd_device_status() == P.OK
    k_sum = additions * U32
    for k in range(G):
        xd, m, r = v[k].double(), mean[k].double().view(B, 1, groups, 1), rstd[k].double().view(B, 1, groups, 1)
        xh = (xd - m) * r
        ga, dz = gamma[k].double().view(groups, D), float(np.float32(0.1))
        # dbeta: the sum's roundings alone; dgamma: each xh is off by the rounding of x - mean and of the product
        want = dz * B * Pn
        assert (dbeta[k].double() - want).abs().max() <= k_sum * want, float((dbeta[k].double() / want - 1).abs().max()) / U32
        size = dz * xh.abs().sum((0, 1)).reshape(C)
        want = dz * xh.sum((0, 1)).reshape(C)
        assert ((dgamma[k].double() - want).abs() <= (k_sum + 3 * U32) * size).all()
        # dx = rstd (gamma dz - m1 - xh m2): m1 and m2 from the same sums, and a handful of roundings of each term
        m1 = dz * ga.mean(1)
        mean_abs = (dz * ga * xh.abs()).mean((1, 3), keepdim=True)
        m2 = (dz * ga * xh).mean((1, 3), keepdim=True)
        tol = r * ((k_sum + 8 * U32) * (m1.view(1, 1, groups, 1) + xh.abs() * mean_abs) + 8 * U32 * dz * ga)
        want = r * (dz * ga - m1.view(1, 1, groups, 1) - xh * m2)
        tol += (U32 if x_type == torch.float32 else 2.0 ** -8) * want.abs()
        off = (dx[k].double().view(B, Pn, groups, D) - want).abs() / tol
        assert off.max() <= 1, float(off.max())


@pytest.mark.gpu
@pytest.mark.parametrize("shape,x_bf16", [((1, 608, 2048, 257, 1), True), ((4, 152, 1100, 1040, 8), True),
                                          ((2, 304, 1500, 1028, 2), False)])
def test_backward_of_many_positions_to_a_thread(P, shape, x_bf16):
    """As many images as leave one range to each, and channels that leave all of its positions to one thread."""
    import torch

    # 64 positions of a segment, its segments, the images by rows of 64, and the ends' trees
    additions = 64 + (shape[2] + 63) // 64 + (shape[1] + 63) // 64 + 16
    _backward(P, shape, torch.bfloat16 if x_bf16 else torch.float32, additions)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, 1 << 20, 1, 8, 1), (3, 300007, 2, 12, 2), (1, 1, 301, 65536, 1), (2, 1, 40, 50000, 1)])
def test_backward_of_many_images_and_of_many_channels_to_a_group(P, shape):
    """The parameters' sums over a worker's images, and a group's means over its channels."""
    import torch

    G, B, Pn, C, groups = shape
    # an image's positions (at most 64 to a thread, then the ranges and the rows of threads), then the longer of: the images by
    # rows of 64, in segments of 64 or of the root of their number (a multiple of 8); the group's channels by lanes of 32, 64 at a
    # time; and the ends' trees
    rows, lanes = -(-B // 64), -(-C // groups // 32)
    seg = max(64, -(-int(rows ** 0.5) // 8) * 8)
    images = min(rows, seg) + -(-rows // seg)
    channels = min(lanes, 64) + -(-lanes // 64)
    _backward(P, shape, torch.float32, min(Pn, 64) + min(Pn, 256) + 8 + max(images, channels) + 16)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,values", [((1, 1, 512, 65536, 1), "two"), ((1, 2, 600, 50001, 1), "two"), ((1, 1, 1200000, 257, 1), "two"),
                                          ((1, 1, 1100000, 1028, 2), "random")])
def test_forward_of_long_merges(P, shape, values):
    """Two alternating values, so that every range and channel has the same moments: their merge over many channels of a
    group, and many segments of positions."""
    import torch

    G, B, Pn, C, groups = shape
    D = C // groups
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(G, B, Pn, C, generator=gen, device="cuda")
    if values == "two":
        x[:, :, 0::2], x[:, :, 1::2] = 0.7, 0.1
    gamma, beta = torch.ones(G, C, device="cuda"), torch.zeros(G, C, device="cuda")
    y = torch.empty_like(x)
    mean, rstd = torch.empty(G * B, groups, device="cuda"), torch.empty(G * B, groups, device="cuda")
    P.lsgd_groupnorm_forward(x, gamma, beta, y, mean, rstd, G, B, Pn, C, groups)
    torch.cuda.synchronize()
    assert P.lsgd_device_status() == P.OK
    # a segment of a thread's positions and its segments (at most 256 ranges or 4096 positions of one), the ranges and channels
    # 64 at a time and the segments of those, and the ends' trees; the variance's relative error is halved by the root
    merges = -(-256 // max(1, 1024 // D)) * -(-D // 1024)
    additions = 2 * max(64, int((Pn / 256) ** 0.5) + 8) + min(merges, 64) + -(-merges // 64) + 24
    for k in range(G):
        xd = x[k].view(B, Pn, groups, D).double()
        m = xd.mean((1, 3))
        r = (xd.var((1, 3), correction=0) + 1e-5).rsqrt()
        big = x[k].abs().max().double()
        dm = additions * U32 * big
        assert ((mean.view(G, B, groups)[k] - m).abs() <= dm).all()
        dr = r * (additions / 2 * U32 + (dm * r) ** 2 + 2 * U32)
        off = ((rstd.view(G, B, groups)[k] - r).abs() / r).max() / U32
        assert ((rstd.view(G, B, groups)[k] - r).abs() <= dr).all(), float(off)
        s = (B, 1, groups, 1)
        z = (xd - m.view(s)) * r.view(s)
        tol = dm * r.view(s) + z.abs() * (dr / r).view(s) + 8 * U32 * (z.abs() + (xd.abs() + m.abs().view(s)) * r.view(s))
        assert ((y[k].view(B, Pn, groups, D) - z).abs() <= tol).all()
