"""Layer norm of rows at the ends of fp32's range: what is promised up to a sum of a row's magnitudes of 3.4e38, and that what lies
beyond stays with its row."""
import numpy as np
import pytest

from test_gpu_layernorm import ACTS, P, ROW, Case  # noqa: F401

# Parts of a warp, a warp, several warps of a CTA, the widest CTA, clusters of 2, 5 and 8
SHAPES = [(2, 9, 5), (1, 40, 100), (2, 9, 777), (1, 6, 4096), (1, 6, 5000), (2, 5, 17000), (1, 4, 32768)]


def _put(c, row, values):
    c.x.rows()[row] = values.to(c.xt)
    return c


# Squared deviations beyond fp32's range, magnitudes that add up to half of it.
@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("shape", SHAPES)
def test_rows_whose_squares_overflow(P, shape, x_type, y_type, act):  # noqa: F811
    import torch

    C = shape[2]
    clean, c = (Case(P, shape, x_type, y_type, act) for _ in range(2))
    clean.forward().backward()
    sign = torch.where(torch.arange(C, device="cuda") % 3 == 0, -1.0, 1.0)
    _put(c, 1, sign * (1.7e38 / C))
    _put(c, 3, torch.full((C,), 1.7e38 / C, device="cuda") * (1 + 0.5 * (torch.arange(C, device="cuda") % 2)))
    c.forward()
    x = c.x.rows()[[1, 3]].double()
    mean = c.mean[[1, 3]].double()
    assert ((mean - x.mean(1)).abs() <= ROW * x.abs().amax(1)).all()
    assert (c.rstd[[1, 3]] == 0).all()
    # y = act(beta): its own roundings alone (SiLU's as in check_forward)
    beta = c.beta[c.pick].view(shape[0], 1, C).expand(shape).reshape(-1, C)[[1, 3]].double()
    want = {"none": beta, "relu": beta.clamp(min=0), "silu": beta * torch.sigmoid(beta)}[act]
    rel = (2.0 ** -8 + 2.0 ** -18) if y_type == "bf16" else 17 * 2.0 ** -24
    assert ((c.y.rows()[[1, 3]].double() - want).abs() <= rel * want.abs() + 1e-37).all()
    c.backward()
    assert (c.dx.rows()[[1, 3]] == 0).all()  # rstd's multiple
    assert torch.isfinite(c.dgamma).all() and torch.isfinite(c.dbeta).all()
    others = torch.tensor([k not in (1, 3) for k in range(c.N)], device="cuda")
    for a, b in ((c.y.rows(), clean.y.rows()), (c.dx.rows(), clean.dx.rows()), (c.mean, clean.mean), (c.rstd, clean.rstd)):
        assert torch.equal(a[others], b[others])


# A sum beyond fp32's range: the row is lost, and no other.
@pytest.mark.gpu
@pytest.mark.parametrize("x_type", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_rows_whose_sum_overflows(P, shape, x_type):  # noqa: F811
    import torch

    clean, c = (Case(P, shape, x_type, x_type, "relu", True) for _ in range(2))
    clean.forward().backward()
    _put(c, 2, torch.full((shape[2],), 3e38, device="cuda"))
    c.forward().backward()
    others = torch.arange(c.N, device="cuda") != 2
    assert not np.isfinite(float(c.mean[2])) and torch.isnan(c.y.rows()[2]).all()
    for a, b in ((c.y.rows(), clean.y.rows()), (c.dx.rows(), clean.dx.rows()), (c.s.rows(), clean.s.rows()), (c.mean, clean.mean),
                 (c.rstd, clean.rstd)):
        assert torch.equal(a[others], b[others])
    assert P.lsgd_device_status() == P.OK
