"""The residual block of test_gpu_block_run.py: what its step gives is finite and, replayed, another draw each time."""
import pytest
import torch

from paper_2412_20796_amd import binding as bd
from test_gpu_block_run import _model, _step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d,dtype", [(1, 64, torch.float32), (640, 128, torch.bfloat16), (301, 200, torch.float16)])
def test_values_of_a_step(rows, d, dtype):
    m = _model(rows, d, dtype)
    step, ws = torch.zeros(1, dtype=torch.int64, device="cuda"), bd.Workspace()
    seen = []
    for k in range(3):
        step.fill_(k)
        r = _step(m, ws, step)
        for name, t in r.items():
            assert bool(torch.isfinite(t.float()).all()), (k, name)
            assert bool(t.any()), (k, name)
        seen.append(r["df"].clone())
    assert rows == 1 or not (torch.equal(seen[0], seen[1]) or torch.equal(seen[1], seen[2]))
