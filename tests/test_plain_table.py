"""CPU: a table's codes and scales."""
import pytest
import torch

from paper_2302_02407_amd.distill import quantize_table


@pytest.mark.parametrize("size", [1.0, 1e30, 1e-30, 1e-37, 1e-39, 1e-42, 1e-44, 0.0])
def test_blocks_of_any_size(size):
    """Codes are numbers, each the nearest to its value: off by 2^-4 of it or 2^-10 of the scale, and where scales are the smallest numbers that 32 bits
    hold by what that rounds them, 448 * 2^-150."""
    w = torch.randn((130, 200), generator=torch.Generator().manual_seed(1))
    w[:128, :128] *= size
    w[3] = 0
    codes, scales = quantize_table(w)
    assert codes.float().isfinite().all() and (codes[3].float() == 0).all()
    back = codes.double() * scales.double().repeat_interleave(128, dim=0)[:130].repeat_interleave(128, dim=1)[:, :200]
    bound = w.double().abs() * 2.0 ** -4 * 1.001 + scales.double().repeat_interleave(128, dim=0)[:130].repeat_interleave(128, dim=1)[:, :200] * 2.0 ** -10 + 450 * 2.0 ** -150
    assert ((back - w.double()).abs() <= bound).all()
