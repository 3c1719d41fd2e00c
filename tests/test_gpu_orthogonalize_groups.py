"""Calls whose matrices go through the workspace in groups."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2601_07876_b200 import ops
    return ops


def test_groups_change_neither_results_nor_what_is_held(ops):
    """Three groups, small matrices between the large ones."""
    torch.manual_seed(0)
    shapes = [(2900, 2900), (40, 50), (2000, 3100), (300, 200)] * 13
    g = [torch.randn(*s, device="cuda", dtype=torch.bfloat16) for s in shapes]
    alone = [ops.orthogonalize(x) for x in g]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    together = ops.orthogonalize(g)
    held = torch.cuda.max_memory_allocated() - before - sum(2 * x.numel() for x in g)
    assert all(torch.equal(a, b) for a, b in zip(alone, together))
    assert held < (1 << 30) + (1 << 24)
    theta, m = [torch.zeros(s, device="cuda") for s in shapes], [torch.zeros(s, device="cuda") for s in shapes]
    ops.orthogonal_step(theta, g, m, [-1.0] * len(g), momentum=0.0, nesterov=False)
    assert all(torch.equal(t.to(torch.bfloat16), a) for t, a in zip(theta, alone))


def test_a_wait_that_runs_out_costs_its_own_group_alone():
    program = os.path.join(os.path.dirname(os.path.abspath(__file__)), "orthogonalize_group_waits.py")
    done = subprocess.run([sys.executable, program], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.count("ok") == 3, done.stdout + done.stderr
