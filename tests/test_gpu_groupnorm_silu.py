"""SiLU's ends: the parameters' gradients are fp32 results for bf16 tensors too, and far negative values."""
import numpy as np
import pytest

from _gpu_common import built_package

U32, U16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


# images of one CTA, of several rounds with the next ones under way, of a cluster, of ranges; one channel to an access
@pytest.mark.gpu
@pytest.mark.parametrize("y_type", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(2, 2, 5, 64, 8), (3000, 1, 4, 64, 8), (1, 4, 1517, 128, 8), (1, 1, 60000, 64, 8), (2, 1, 5, 63, 9)])
def test_parameter_gradients_of_bf16_tensors(P, shape, y_type):
    """gamma = 0, so that z = beta exactly, and dy = 1 at one position of each worker, so that nothing is added: dbeta is SiLU's
    slope at beta, dgamma that times xh."""
    import torch

    G, B, Pn, C, groups = shape
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(G, B, Pn, C, generator=gen, device="cuda").bfloat16()
    gamma = torch.zeros(G, C, device="cuda")
    beta = -1.5 - 80 * torch.rand(G, C, generator=gen, device="cuda")
    dy = torch.zeros(G, B, Pn, C, dtype=torch.bfloat16 if y_type == "bf16" else torch.float32, device="cuda")
    dy[:, B - 1, Pn // 2] = 1
    v = x.double().view(G, B, Pn, groups, C // groups)
    mean, rstd = v.mean((2, 4)).float(), (v.var((2, 4), correction=0) + 1e-5).rsqrt().float()
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
    P.lsgd_groupnorm_backward(x, None, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, G, B, Pn, C, groups, act=P.ACT_SILU)
    torch.cuda.synchronize()
    assert P.lsgd_device_status() == P.OK
    z = beta.double()
    s = 1 / (1 + torch.exp(-z))
    inner = 1 + z * (1 - s)
    want = s * inner
    # s: the exponential's 2 units in the last place (4 halves), the sum, and the reciprocal's 2^-23; 1 - s and the fused sum with
    # z, then the product (dz = dy times it is exact)
    tol = U32 * (7 * want.abs() + s * (z.abs() * (1 + 7 * s) + inner.abs()) + 2 * want.abs()) * 1.01
    off = ((dbeta.double() - want).abs() / tol).max()
    assert off <= 1, float(off)
    m, r = (t.view(G, B, groups)[:, B - 1].double().repeat_interleave(C // groups, 1) for t in (mean, rstd))
    xh = (x[:, B - 1, Pn // 2].double() - m) * r
    off = ((dgamma.double() - want * xh).abs() / (tol * xh.abs() + 4 * U32 * (want * xh).abs())).max()
    assert off <= 1, float(off)


@pytest.mark.gpu
@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("shape", [(1, 2, 64, 64, 8), (1, 1, 60000, 64, 8), (700, 2, 16, 64, 4)])
def test_far_negative_values(P, shape, x_type, y_type):
    """z between -110 and -60: y is the function's value, or 0 where that is below 1e-36 (the exponential's end)."""
    import torch

    G, B, Pn, C, groups = shape
    t = {"bf16": torch.bfloat16, "fp32": torch.float32}
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(G, B, Pn, C, generator=gen, device="cuda").to(t[x_type])
    gamma, beta = torch.ones(G, C, device="cuda"), -65 - 40 * torch.rand(G, C, generator=gen, device="cuda")
    y = torch.empty(G, B, Pn, C, dtype=t[y_type], device="cuda")
    mean, rstd = torch.empty(G * B, groups, device="cuda"), torch.empty(G * B, groups, device="cuda")
    P.lsgd_groupnorm_forward(x, gamma, beta, y, mean, rstd, G, B, Pn, C, groups, act=P.ACT_SILU)
    torch.cuda.synchronize()
    v = x.double().view(G, B, Pn, groups, C // groups)
    z = ((v - mean.double().view(G, B, 1, groups, 1)) * rstd.double().view(G, B, 1, groups, 1)).view(x.shape)
    z = z + beta.double().view(G, 1, 1, C)
    want = z / (1 + torch.exp(-z))
    # z is off by 4 roundings of its terms, which the exponential turns into as much of the value; and the function's own
    rel = 4 * U32 * (z.abs() + beta.double().abs().view(G, 1, 1, C) + 8) + (16 * U32 if y_type == "fp32" else 2.0 ** -15)
    tol = (rel + (U32 if y_type == "fp32" else U16)) * want.abs() + 1.1e-36
    got = y.double()
    assert ((got - want).abs() <= tol).all(), float(((got - want).abs() / tol).max())
    assert (got <= 0).all() and torch.isfinite(got).all()
