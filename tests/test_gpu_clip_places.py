"""Clipping to places that share a buffer with what is read: every worker's values come out once, where they belong."""
import numpy as np
import pytest

from _gpu_common import built_package


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


def _types(torch, name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def _fill(torch, views, seed):
    """Workers by turns below and above a norm of 1 (the first of them below)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = sum(v.shape[1] for v in views)
    G = views[0].shape[0]
    scale = torch.tensor([(0.5, 2.0)[k % 2] for k in range(G)], device="cuda")[:, None] / n ** 0.5
    for v in views:
        v.copy_(torch.randn(v.shape, generator=gen, device="cuda") * scale)


def _factor(torch, norm, limit=1.0):
    """The clipping factor's fp32 quotient (a number over a tensor is its reciprocal's multiple in torch, rounded twice)."""
    return torch.clamp(torch.full_like(norm, limit) / norm, max=1.0)[:, None]


# The first worker's place is where it was read, the others' are not.  Sizes of one launch, of two, and of one CTA to a worker; the
# workers' values further apart than they were, and closer together.
@pytest.mark.gpu
@pytest.mark.parametrize("G,n", [(3, 100), (4, 777), (4, 300_001), (700, 50)])
@pytest.mark.parametrize("apart", [True, False])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_first_place_in_common(P, G, n, apart, dtype):
    import torch

    t = _types(torch, dtype)
    near, far = n, G * n  # near workers stand within the first far one's stride
    buf = torch.full((far * (G - 1) + n + 8,), 77.0, device="cuda", dtype=t)
    close, wide = buf.as_strided((G, n), (near, 1)), buf.as_strided((G, n), (far, 1))
    g, out = (close, wide) if apart else (wide, close)
    other = torch.empty(G, 33, device="cuda", dtype=t)
    _fill(torch, [g, other], n)
    held, held_other = g.clone(), other.clone()
    other_out = torch.full_like(other, 77.0)
    norm = torch.empty(G, device="cuda")
    P.lsgd_gradient_clip(P.lsgd_tensors_create([g, other], [out, other_out]), norm, 1.0)
    torch.cuda.synchronize()
    low = norm <= 1
    assert low.any() and not low.all() and bool(low[0])
    f = _factor(torch, norm)
    want = (held.float() * f).to(t)
    assert torch.equal(want[low], held[low])
    for k in range(G):
        assert torch.equal(out[k], want[k]), k
    assert torch.equal(other_out, (held_other.float() * f).to(t))
    # what was read stands as it was, where nothing was written over it
    assert torch.equal(g[1:], held[1:])


# Worker 0 clipped too: the same layout where no worker is left as it is, and where all are.
@pytest.mark.gpu
@pytest.mark.parametrize("limit", [1e-3, 1e3])
def test_the_first_place_in_common_as_rows_of_a_buffer(P, limit):
    import torch

    buf = torch.randn(6, 100, device="cuda")
    g, out = buf[:2], buf[::3]
    held = g.clone()
    norm = torch.empty(2, device="cuda")
    P.lsgd_gradient_clip(P.lsgd_tensors_create([g], [out]), norm, limit)
    torch.cuda.synchronize()
    assert torch.equal(out, held * _factor(torch, norm, limit)) and torch.equal(buf[1], held[1])


# Layouts that a list may have, by (first value, workers' stride) in one buffer of values of a type, where what is written meets nothing
# else: they are taken, and every value comes out as if it stood alone.  None: clipped in place.
LAYOUTS = {
    "pieces of one buffer, in place": [((0, 200), None, 100), ((100, 200), None, 100)],
    "in place by name": [((0, 200), (0, 200), 100)],
    "in place by name, beside others": [((0, 200), (0, 200), 100), ((100, 200), (1000, 100), 100)],
    "read twice, written apart": [((0, 100), (1000, 100), 100), ((0, 100), (2000, 100), 100)],
    "read twice in part, written apart": [((0, 150), (1000, 150), 150), ((50, 150), (2000, 100), 100)],
    "written between what is read": [((0, 300), (100, 300), 100), ((200, 300), (1000, 100), 100)],
    "written into the gaps of what is written": [((1000, 100), (0, 300), 100), ((2000, 100), (100, 300), 100), ((3000, 100), (200, 300), 100)],
    "pieces that end where the next begins, written the other way round": [((0, 64), (2031, 64), 33), ((33, 64), (2000, 64), 31)],
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(LAYOUTS))
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("times", [1, 1001])
def test_layouts_that_are_taken(P, name, dtype, times):
    import torch

    G, t = 3, _types(torch, dtype)
    layout = [(i, o, n) for i, o, n in LAYOUTS[name]]
    buf = torch.full((4000 * times,), 77.0, device="cuda", dtype=t)
    at = lambda place, n: buf.as_strided((G, n * times), (place[1] * times, 1), place[0] * times)  # noqa: E731
    grads = [at(i, n) for i, _, n in layout]
    _fill(torch, grads, times)
    outs = None if layout[0][1] is None else [at(o, n) for _, o, n in layout]
    held, before = [g.clone() for g in grads], buf.clone()
    norm = torch.empty(G, device="cuda")
    limit = float(sum((g[0].double() ** 2).sum() for g in grads) ** 0.5 * 1.01)  # workers 0 and 2 below it
    P.lsgd_gradient_clip(P.lsgd_tensors_create(grads, outs), norm, limit)
    torch.cuda.synchronize()
    want_norm = sum((h.double() ** 2).sum(1) for h in held).sqrt()
    assert ((norm.double() - want_norm).abs() <= 37 * 2.0 ** -24 * want_norm).all()
    f, want = _factor(torch, norm, limit), before
    assert bool(f[0] == 1) and bool(f[1] < 1)
    for h, (i, o, n) in zip(held, layout):
        want.as_strided((G, n * times), ((o or i)[1] * times, 1), (o or i)[0] * times).copy_((h.float() * f).to(t))
    assert torch.equal(buf, want)
