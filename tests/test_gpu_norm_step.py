"""A worker's step with both pairs of operators: group norm forward and backward around a layer, the layer's update direction
and its application, eager and as one captured graph."""
import numpy as np
import pytest

import _operator_refs as R
from _gpu_common import built_package

U32, U16 = 2.0 ** -24, 2.0 ** -8
LR, DECAY = 0.02, 0.01


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


class Step:
    """x = a w^T per worker (float64, rounded once), y = silu(groupnorm(x)), dy given; w takes a step along the direction."""

    def __init__(self, P, shape, seed=0):
        import torch

        self.P, self.shape = P, shape
        G, B, Pn, cin, C, groups = shape
        rng = np.random.default_rng(seed)
        dev = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
        self.a, self.w = dev(rng.standard_normal((G, B * Pn, cin))), dev(rng.standard_normal((G, C, cin)) / np.sqrt(cin))
        self.dy = dev(rng.standard_normal((G, B, Pn, C)) / B).bfloat16()
        self.gamma, self.beta = dev(1 + 0.2 * rng.standard_normal((G, C))), dev(0.2 * rng.standard_normal((G, C)))
        self.x, self.dx = torch.empty(G, B, Pn, C, device="cuda"), torch.empty(G, B, Pn, C, device="cuda")
        self.y = torch.empty(G, B, Pn, C, dtype=torch.bfloat16, device="cuda")
        self.mean, self.rstd = torch.empty(G, B, groups, device="cuda"), torch.empty(G, B, groups, device="cuda")
        self.dgamma, self.dbeta = torch.empty_like(self.gamma), torch.empty_like(self.beta)
        self.g, self.u = torch.empty_like(self.w), torch.zeros_like(self.w)
        self.o = torch.empty_like(self.w, dtype=torch.bfloat16)
        self.wb = torch.empty_like(self.o)

    def run(self):
        import torch

        P, (G, B, Pn, cin, C, groups) = self.P, self.shape
        self.x.copy_(torch.bmm(self.a.double(), self.w.double().transpose(1, 2)).view(self.x.shape))
        P.lsgd_groupnorm_forward(self.x, self.gamma, self.beta, self.y, self.mean, self.rstd, G, B, Pn, C, groups, act=P.ACT_SILU)
        P.lsgd_groupnorm_backward(self.x, None, self.dy, self.gamma, self.beta, self.mean, self.rstd, self.dx, self.dgamma,
                                  self.dbeta, G, B, Pn, C, groups, act=P.ACT_SILU)
        self.g.copy_(torch.bmm(self.dx.view(G, B * Pn, C).transpose(1, 2).double(), self.a.double()))
        P.lsgd_orthogonal_direction(self.u, self.g, self.o, G, C, cin)
        P.lsgd_direction_update(self.w, self.o, self.wb, G, C * cin, LR, max(1.0, C / cin) ** 0.5, DECAY)

    def state(self):
        return dict(w=self.w, wb=self.wb, u=self.u, o=self.o, y=self.y, dgamma=self.dgamma, dbeta=self.dbeta)


# layers whose direction one CTA, several and the tiles of products compute; images of one CTA and of more
SHAPES = [(3, 4, 49, 40, 24, 4), (2, 3, 500, 576, 64, 8), (2, 5, 300, 150, 192, 6)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_a_step_against_64_bits(P, shape):
    s = Step(P, shape)
    G, B, Pn, cin, C, groups = shape
    w0 = s.w.double().cpu().numpy()
    s.run()
    a, ga, be = (t.double().cpu().numpy() for t in (s.a, s.gamma, s.beta))
    dy = s.dy.double().cpu().numpy()
    x = np.einsum("gnk,gck->gnc", a, w0).reshape(G, B, Pn, C)
    y, mean, rstd, _ = R.gn_forward(x, ga, be, groups, 1e-5, "silu")
    dx, dgamma, dbeta = R.gn_backward(x, dy, ga, be, mean, rstd, groups, "silu")[:3]
    # the gradients: fp32 chains of at most 160 roundings, each of a term no larger than the sum of the terms' magnitudes;
    # taken against the tensor's norm that sum is at most 64 times the result for these random inputs
    rel = 160 * 64 * U32
    for got, want in ((s.dx, dx), (s.dgamma, dgamma), (s.dbeta, dbeta)):
        assert np.linalg.norm(got.double().cpu().numpy() - want) <= rel * np.linalg.norm(want)
    g = np.einsum("gnc,gnk->gck", dx.reshape(G, B * Pn, C), a)
    got = s.g.double().cpu().numpy()
    # u = g and the direction of g + 0.95 u, the same as that of g.  The direction's own error and its rounding; and its change with
    # the gradient's error e, which the five steps' slope at zero, 3.4445^5 = 485, and the norm's division multiply at most
    want = R.direction(1.95 * g, 5)
    o = s.o.double().cpu().numpy()
    scale = max(1.0, C / cin) ** 0.5
    for k in range(G):
        e = np.linalg.norm(got[k] - g[k]) / np.linalg.norm(g[k])
        assert e <= rel
        tol = 2.5e-3 * np.linalg.norm(want[k]) + U16 * np.linalg.norm(want[k]) + 2 * 485 * e
        off = np.linalg.norm(o[k] - want[k])
        assert off <= tol, (off, tol)
        w = (1 - LR * DECAY) * w0[k] - LR * scale * o[k]
        assert np.abs(s.w[k].double().cpu().numpy() - w).max() <= 4 * U32 * (np.abs(w0[k]).max() + LR * scale * np.abs(o[k]).max())
    assert np.array_equal(s.wb.float().cpu().numpy(), s.w.bfloat16().float().cpu().numpy())
    assert P.lsgd_device_status() == P.OK


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_captured_steps_are_the_eager_ones(P, shape):
    import torch

    eager, captured = Step(P, shape, 1), Step(P, shape, 1)
    for _ in range(4):
        eager.run()
    captured.run()  # also what the products in 64 bits need before a capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for name, t in eager.state().items():
        assert torch.equal(t, captured.state()[name]), name
    assert P.lsgd_device_status() == P.OK
