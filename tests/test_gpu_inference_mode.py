"""Tensors made in inference mode may not be written over outside of it: the error comes before they change."""
import pytest
import torch

import paper_2202_13808_b200 as dropit

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", [0, 1])
def test_rotation_in_place(cuda_device, which):
    plan, at = dropit.dropit_rotary_plan(16, (16,)), torch.arange(1, 5, device=cuda_device).unsqueeze(1)
    draw = lambda: torch.randn(2, 4, 3, 16, device=cuda_device)
    with torch.inference_mode():
        kept = draw()
        inside = dropit.dropit_rotary(kept.clone(), None, at, plan, in_place=True)[0]
    pair = [draw(), draw()]
    pair[which] = kept
    before = [t.clone() for t in pair]
    with torch.no_grad(), pytest.raises(RuntimeError, match="inference"):
        dropit.dropit_rotary(*pair, at, plan, in_place=True)
    assert torch.equal(kept, before[which])
    assert torch.equal(dropit.dropit_rotary(kept, None, at, plan)[0], inside)
