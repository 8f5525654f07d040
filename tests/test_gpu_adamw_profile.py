"""The step under a profiler."""
import pytest
import torch

import paper_2202_13808_b200 as dropit

pytestmark = pytest.mark.gpu


def test_a_step_has_its_label_in_a_trace(cuda_device):
    p = torch.nn.Parameter(torch.ones(8, device=cuda_device))
    opt = dropit.DropITAdamW([p], lr=1e-2)
    p.grad = torch.ones_like(p)
    opt.step()
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as trace:
        opt.step()
    assert any("DropITAdamW" in e.key for e in trace.key_averages())
    assert int(opt.state[p]["step"]) == 2
