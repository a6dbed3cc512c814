"""Clipping factors at and beyond the ends of fp32's range, against 64 bits."""
import numpy as np
import pytest

from _gpu_common import built_package

U32, U16 = 2.0 ** -24, 2.0 ** -8  # largest relative roundings of fp32 and bf16
# The norm's: a value's square passes 66 roundings in a lane and 5 between lanes, halved by the root, whose own and that to fp32 follow.
NORM = 37 * U32
FACTOR = NORM + 3 * U32  # the quotient's, the product's, the limit's


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


def _types(torch, name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def _norm64(g):
    return (g.double() ** 2).sum(1).sqrt()


def _close(torch, got, want, rel):
    """A result of factors and products within `rel`, and the rounding to its type (2^-149 and 2^-133 apart at the bottom)."""
    bf16 = got.dtype == torch.bfloat16
    tol = (rel + (U16 if bf16 else U32)) * want.abs() + (2.0 ** -133 if bf16 else 2.0 ** -149)
    return bool(((got.double() - want).abs() <= tol).all())


# One launch, two, one CTA to a worker (its sum of squares is not kept).
FORMS = [(2, 10_000), (2, 300_001), (700, 2000)]
TYPES = [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "fp32")]


def _clip_both_ways(P, G, n, types, scale, limit, others):
    """Worker 1 at `scale`, the others at `others`: to places of another alignment, and in place."""
    import torch

    a, b = (_types(torch, t) for t in types)
    gen = torch.Generator(device="cuda").manual_seed(n)
    size = torch.full((G, 1), others, device="cuda", dtype=torch.float64)
    size[1] = scale
    buf = torch.zeros(G, n + 3, device="cuda", dtype=a)
    g = buf[:, 1:n + 1]
    g.copy_(torch.randn(G, n, generator=gen, device="cuda", dtype=torch.float64) * size)
    want_norm = _norm64(g)
    want = g.double() * torch.clamp(limit / want_norm, max=1.0)[:, None]
    obuf = torch.full((G, n + 9), 77.0, device="cuda", dtype=b)
    norm = torch.empty(G, device="cuda")
    held = g.clone()
    for out in (obuf[:, 2:n + 2], obuf[:, 1:n + 1]):
        obuf.fill_(77.0)
        P.lsgd_gradient_clip(P.lsgd_tensors_create([g], [out]), norm, limit)
        torch.cuda.synchronize()
        assert _close(torch, out, want, FACTOR)
        assert int((obuf == 77).sum()) >= obuf.numel() - out.numel() and torch.equal(g, held)
    if a == b:
        P.lsgd_gradient_clip(P.lsgd_tensors_create([g]), norm, limit)
        torch.cuda.synchronize()
        assert _close(torch, g, want, FACTOR)
    return norm, want_norm


# Factors of 1e-40 and less, which fp32 holds with few bits or not at all, while their products are ordinary numbers.
@pytest.mark.gpu
@pytest.mark.parametrize("G,n", FORMS)
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("scale,limit", [(1e34, 1e-5), (1e34, 1e-12), (1e30, 1e-30), (1e20, 3e-38)])
def test_small_factors_keep_their_bits(P, G, n, types, scale, limit):
    norm, want = _clip_both_ways(P, G, n, types, scale, float(np.float32(limit)), scale)
    assert bool(((norm.double() - want).abs() <= NORM * want).all())


# Finite gradients whose norm passes fp32's range (and is infinite as it is given) are clipped by the norm that they have.
@pytest.mark.gpu
@pytest.mark.parametrize("G,n", FORMS)
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("limit", [3e38, 1.0, 1e-30])
def test_norms_beyond_fp32(P, G, n, types, limit):
    norm, want = _clip_both_ways(P, G, n, types, 2e37, float(np.float32(limit)), 1.0)
    ordinary = norm[[k for k in range(G) if k != 1]].double()
    assert bool(norm[1] == float("inf")) and float(want[1]) > 4e38
    assert bool(((ordinary - want[[k for k in range(G) if k != 1]]).abs() <= NORM * ordinary).all())


@pytest.mark.gpu
def test_norms_beyond_fp32_of_several_types(P):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(1)
    grads = [(torch.randn(3, n, generator=gen, device="cuda", dtype=torch.float64) * 3e37).to(t)
             for n, t in ((5000, torch.float32), (777, torch.bfloat16), (3, torch.float32))]
    grads[0][2, 4] = float("inf")
    squares = sum(_norm64(g) ** 2 for g in grads)
    outs, norm = [torch.empty_like(g) for g in grads], torch.empty(3, device="cuda")
    P.lsgd_gradient_clip(P.lsgd_tensors_create(grads, outs), norm, 5.0)
    torch.cuda.synchronize()
    assert bool((norm == float("inf")).all())
    for g, o in zip(grads, outs):
        assert _close(torch, o[:2], g[:2].double() * (5.0 / squares[:2].sqrt())[:, None], FACTOR)
    # an infinite value: zeros, and its own product NaN
    assert bool(torch.isnan(outs[0][2, 4])) and bool((outs[1][2] == 0).all()) and bool((outs[0][2, 5:] == 0).all())


# Small factors of the update: w = 0, so that w = -lr g' shows the clipped gradient.  Vectors, and single values at odd strides.
@pytest.mark.gpu
@pytest.mark.parametrize("g_type", ["fp32", "bf16"])
@pytest.mark.parametrize("n,stride", [(1000, 1000), (1001, 1003)])
@pytest.mark.parametrize("scale,limit", [(1e35, 1e-5), (1e35, 1e-7), (1e20, 1e-30), (1e34, 1e-12)])
def test_small_factors_of_the_update(P, n, stride, g_type, scale, limit):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(n)
    buf = torch.zeros(3, stride, device="cuda", dtype=_types(torch, g_type))
    g = buf[:, :n]
    g.copy_(torch.randn(3, n, generator=gen, device="cuda", dtype=torch.float64) * scale)
    norm = _norm64(g).float()
    w, u = torch.zeros(3, n, device="cuda"), torch.zeros(3, n, device="cuda")
    limit = float(np.float32(limit))
    P.lsgd_clipped_update(w, u, buf, None, 3, n, norm, limit, 0.5, momentum=0.75, g_gs=stride)
    torch.cuda.synchronize()
    want = g.double() * (limit / norm.double())[:, None]
    assert _close(torch, u, want, 3 * U32) and _close(torch, w, -0.5 * want, 3 * U32)
