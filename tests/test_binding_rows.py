"""binding._rows: which layouts of a row tensor are taken (the check comes before a device is asked for)."""
import pytest
import torch

from paper_2506_05413_b200 import binding


@pytest.mark.parametrize("t", [torch.zeros(8, 2).T[:1], torch.zeros(1, 16)[:, ::2], torch.zeros(1, 1).expand(1, 8),
                               torch.zeros(8, 2).T, torch.zeros(2, 16)[:, ::2], torch.zeros(8), torch.zeros(1, 2, 4)])
def test_rows_whose_values_are_not_neighbours_are_refused(t):
    with pytest.raises(ValueError):
        binding._rows(t, t.dtype, "t")


@pytest.mark.parametrize("t", [torch.zeros(3, 16)[1:2, :8], torch.zeros(3, 16)[:, 4:12], torch.zeros(1, 8), torch.zeros(8, 1).T,
                               torch.zeros(0, 16)[:, ::2], torch.zeros(5, 1)])
def test_other_rows_reach_the_device_check(t):
    with pytest.raises(TypeError):
        binding._rows(t, t.dtype, "t")
