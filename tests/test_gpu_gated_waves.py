"""dx where the last wave of tiles is nearly empty and its rows become a launch of their own."""
import pytest
import torch

import paper_2202_13808_b200 as dropit

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tiles_over", [1, 2, 3])
def test_rows_behind_the_full_waves(cuda_device, tiles_over):
    """256 x 256 tiles on about 74 pairs of SMs: enough rows for every count of pairs from 60 to 80 to leave a few tiles over somewhere, and a ragged end."""
    C, H = 256, 64
    g = torch.Generator(device=cuda_device).manual_seed(tiles_over)
    w = (torch.randn(2 * H, C, generator=g, device=cuda_device) * C ** -0.5).bfloat16()
    pairs = torch.cuda.get_device_properties(cuda_device).multi_processor_count // 2
    for waves in (1, 2):
        for less in range(0, 5):        # some SMs may have no partner
            M = 256 * (waves * (pairs - less) + tiles_over) - 37
            dgu = torch.randn(M, 2 * H, generator=g, device=cuda_device).bfloat16()
            dx = dropit.dropit_gated_input_grad(dgu, w)
            want, size = dgu.double() @ w.double(), dgu.double().abs() @ w.double().abs()
            bound = 2 * H * 2.0 ** -24 * size
            assert bool(((dx.double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all())
    dropit.check_device_status(cuda_device)
