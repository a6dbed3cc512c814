"""The norm of a large matrix of equal magnitudes, whose squares' roundings all go one way."""
import numpy as np
import pytest

from _gpu_common import built_package


@pytest.mark.gpu
@pytest.mark.parametrize("momentum", [0.0, 0.5])
def test_norm_of_a_large_matrix_of_equal_magnitudes(momentum):
    """One step on values +-c: o = (a S + (b A + c A A) S) / ||S|| for the signs S is near a / sqrt(rows cols), which lies 1e-5
    from the middle between two bf16 values at this size, with a spread from A's off-diagonals: rows of them, each of
    1 / (rows sqrt(cols)) in the mean, make sqrt(rows) / (rows sqrt(cols)) b / a = 6.4e-5 x 1.39 = 8.8e-5 of it.  An error e of
    the norm puts 0.4 e / 8.8e-5 of the values on the other side of that middle: 11 % for the 2.5e-5 of sums of 3778 squares
    in a row.  Sums of 64, then of 60, 8 and the ends' trees are off by at most 64 + 60 + 8 + 18 roundings of 2^-24, half of that
    in the norm: 4.5e-6, and 1e-6 from the values' own arithmetic, 2.5 %."""
    import torch

    P = built_package()
    rows, cols, c = 16384, 15112, float(np.float32(0.3107))
    gen = torch.Generator(device="cuda").manual_seed(5)
    S = torch.randint(0, 2, (rows, cols), generator=gen, device="cuda", dtype=torch.float32).mul_(2).sub_(1)
    g = S * c
    u = torch.zeros_like(g) if momentum else None
    o = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    P.lsgd_orthogonal_direction(u, g, o, 1, rows, cols, momentum=momentum, nesterov=False, steps=1)
    torch.cuda.synchronize()
    assert P.lsgd_device_status() == P.OK
    # whole numbers: S S^T is exact in fp32, (S S^T) S to a unit or so of its 5e4
    SS = S @ S.t()
    first = SS @ S
    second = SS @ first
    n2 = float(rows) * cols
    a, b, cc = (float(np.float32(v)) for v in (3.4445, -4.7750, 2.0315))
    want = (a * S.double() + (b / n2) * first.double() + (cc / n2 ** 2) * second.double()) / n2 ** 0.5
    other = (o != want.bfloat16()).double().mean().item()
    spread = (want.abs().std() / want.abs().mean()).item()
    assert 7e-5 < spread < 1.1e-4 and (want.abs().bfloat16().unique().numel() > 1)
    assert other < 0.025, other
