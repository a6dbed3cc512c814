"""A worker's step on rows with the operators together: a dense layer with a residual, layer norm forward and backward, the norm of the
whole gradient, the update clipped by it; eager and as one captured graph."""
import numpy as np
import pytest

import _operator_refs as R
from _gpu_common import built_package

U32 = 2.0 ** -24
LR, DECAY, MOMENTUM = 0.05, 0.01, 0.9


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


class Step:
    """s = a w^T + r per worker (the product in float64, rounded once), y = silu(layernorm(s)), dy and ds given.  A worker's w, gamma and
    beta stand in one replica-major buffer, as their momenta, gradients and bf16 copies do."""

    def __init__(self, P, shape, seed=0):
        import torch

        self.P, self.shape = P, shape
        G, Rn, cin, C = shape
        rng = np.random.default_rng(seed)
        dev = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
        self.d = C * cin + 2 * C
        self.pad = (self.d + 63) // 64 * 64
        par = np.zeros((G, self.pad))
        par[:, :C * cin] = rng.standard_normal((G, C * cin)) / np.sqrt(cin)
        par[:, C * cin:C * cin + C] = 1 + 0.2 * rng.standard_normal((G, C))
        par[:, C * cin + C:self.d] = 0.2 * rng.standard_normal((G, C))
        self.w, self.u, self.g = dev(par), dev(np.zeros((G, self.pad))), dev(np.zeros((G, self.pad)))
        self.wb = torch.zeros(G, self.pad, dtype=torch.bfloat16, device="cuda")
        self.a, self.r = dev(rng.standard_normal((G, Rn, cin))), dev(rng.standard_normal((G, Rn, C)))
        self.dy, self.ds = dev(rng.standard_normal((G, Rn, C)) / Rn), dev(rng.standard_normal((G, Rn, C)) / Rn)
        self.x, self.s, self.y, self.dx = (torch.empty(G, Rn, C, device="cuda") for _ in range(4))
        self.mean, self.rstd, self.norm = torch.empty(G, Rn, device="cuda"), torch.empty(G, Rn, device="cuda"), torch.empty(G, device="cuda")
        n = C * cin
        self.list = P.lsgd_tensors_create([self.g[:, :n], self.g[:, n:n + C], self.g[:, n + C:self.d]])

    def run(self, max_norm):
        import torch

        P, (G, Rn, cin, C) = self.P, self.shape
        n = C * cin
        w = self.w[:, :n].unflatten(1, (C, cin))
        self.x.copy_(torch.bmm(self.a.double(), w.double().transpose(1, 2)))
        flat = lambda t, at: t.view(-1)[at:]  # noqa: E731
        kw = dict(act=P.ACT_SILU, par_gs=self.pad)
        P.lsgd_layernorm_forward(self.x, flat(self.w, n), flat(self.w, n + C), self.y, self.mean, self.rstd, G, Rn, C, r=self.r, s=self.s,
                                 **kw)
        P.lsgd_layernorm_backward(self.s, None, self.dy, flat(self.w, n), flat(self.w, n + C), self.mean, self.rstd, self.dx,
                                  flat(self.g, n), flat(self.g, n + C), G, Rn, C, ds=self.ds, **kw)
        self.g[:, :n].unflatten(1, (C, cin)).copy_(torch.bmm(self.dx.double().transpose(1, 2), self.a.double()))
        P.lsgd_gradient_norm(self.list, self.norm)
        P.lsgd_clipped_update(self.w, self.u, self.g, self.wb, G, self.d, self.norm, max_norm, LR, MOMENTUM, True, DECAY, decay_end=n,
                              w_gs=self.pad, g_gs=self.pad)

    def state(self):
        return dict(w=self.w, u=self.u, wb=self.wb, g=self.g, y=self.y, s=self.s, norm=self.norm, dx=self.dx)


SHAPES = [(3, 20, 24, 40), (2, 300, 65, 513), (1, 90, 40, 5000)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_a_step_against_64_bits(P, shape):
    s = Step(P, shape)
    G, Rn, cin, C = shape
    n = C * cin
    w0 = s.w.double().cpu().numpy()
    a, r, dy, ds = (t.double().cpu().numpy() for t in (s.a, s.r, s.dy, s.ds))
    ga, be = w0[:, n:n + C], w0[:, n + C:s.d]
    x = np.einsum("grk,gck->grc", a, w0[:, :n].reshape(G, C, cin)) + r
    row = lambda t: t.reshape(G, Rn, 1, C)  # noqa: E731
    y, mean, rstd, _ = R.gn_forward(row(x), ga, be, 1, 1e-5, "silu")
    dx, dg, db = R.gn_backward(row(x), row(dy), ga, be, mean, rstd, 1, "silu")[:3]
    dx = dx.reshape(G, Rn, C) + ds
    g = np.concatenate([np.einsum("grc,grk->gck", dx, a).reshape(G, n), dg, db], 1)
    norm = np.linalg.norm(g, axis=1)
    limit = float(np.float32(0.5 * norm.min()))
    s.run(limit)
    # fp32 chains of at most 160 roundings of terms no larger than the sums of their magnitudes, which for these random inputs are at
    # most 64 times the results' 2-norms
    rel = 160 * 64 * U32
    close = lambda got, want: np.linalg.norm(got - want) <= rel * np.linalg.norm(want)  # noqa: E731
    got = {k: v.double().cpu().numpy() for k, v in s.state().items()}
    assert close(got["y"], y.reshape(G, Rn, C)) and close(got["dx"], dx) and close(got["s"], x)
    assert close(got["g"][:, :s.d], g) and (np.abs(got["norm"] - norm) <= rel * norm).all()
    f = limit / norm[:, None]
    step = f * g
    step[:, :n] += DECAY * w0[:, :n]
    assert close(got["u"][:, :s.d], step)
    w = w0[:, :s.d] - LR * (1 + MOMENTUM) * step
    assert np.abs(got["w"][:, :s.d] - w).max() <= rel * LR * 2 * np.abs(step).max() + 4 * U32 * np.abs(w).max()
    assert np.array_equal(got["wb"][:, :s.d], s.w.bfloat16().double().cpu().numpy()[:, :s.d])
    # the clipped gradients have the norm that they were clipped to
    out = P.lsgd_tensors_create([s.g[:, :n], s.g[:, n:s.d]])
    P.lsgd_gradient_clip(out, s.norm, limit)
    P.lsgd_gradient_norm(out, s.norm)
    assert (np.abs(s.norm.cpu().numpy() / limit - 1) <= 80 * U32).all()  # two norms, a product's rounding
    assert P.lsgd_device_status() == P.OK


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_captured_steps_are_the_eager_ones(P, shape):
    import torch

    eager, captured = Step(P, shape, 1), Step(P, shape, 1)
    for _ in range(4):
        eager.run(0.7)
    captured.run(0.7)  # also what the products in 64 bits need before a capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run(0.7)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for name, t in eager.state().items():
        assert torch.equal(t, captured.state()[name]), name
    assert P.lsgd_device_status() == P.OK
