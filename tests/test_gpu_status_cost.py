"""lsgd_device_status asks the kernels of an operator for their flag only once the operator has been called."""
import json
import os
import subprocess
import sys

import pytest

from _gpu_common import built_package

SCRIPT = """
import json, statistics, time
import torch
import paper_1808_07217_gb300 as P

def cost():
    def once():
        t = time.perf_counter()
        assert P.lsgd_device_status() == P.OK
        return time.perf_counter() - t
    for _ in range(50):
        once()
    return statistics.median(once() for _ in range(1000))

torch.zeros(1, device="cuda")
out = [cost()]
x, one = torch.randn(1, 2, 16, 64, device="cuda"), torch.ones(1, 64, device="cuda")
stats = torch.empty(2, 2, 8, device="cuda")
P.lsgd_groupnorm_forward(x, one, one.clone(), torch.empty_like(x), stats[0], stats[1], 1, 2, 16, 64, 8)
out.append(cost())
g = torch.randn(1, 16, 64, device="cuda")
P.lsgd_orthogonal_direction(None, g, torch.empty_like(g, dtype=torch.bfloat16), 1, 16, 64, momentum=0.0)
out.append(cost())
print(json.dumps(out))
"""


@pytest.mark.gpu
def test_status_without_the_operators_costs_what_it_did():
    built_package()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", SCRIPT], cwd=root, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
    none, norm, both = json.loads(run.stdout.splitlines()[-1])
    # one copy of a flag, then two, then three, which take most of the call
    assert none < 0.7 * both and norm < 0.9 * both, (none, norm, both)
