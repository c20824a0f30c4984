"""What the binding keeps between calls: numbers only."""
import torch

from paper_2102_04782_amd import binding as daq


def test_a_scale_held_in_a_tensor_is_read_at_every_call():
    scale = torch.tensor(2.0)
    assert daq._route_opts(daq.SCORES_SIGMOID, 2, 1, 1, True, scale).scale == 2.0
    scale.fill_(3.0)
    assert daq._route_opts(daq.SCORES_SIGMOID, 2, 1, 1, True, scale).scale == 3.0
