"""A stream of another device than the call's tensors is refused: the work would have gone to some other stream of theirs (no GPU needed)."""
import pytest
import torch

from paper_2505_01572_amd import binding, operators


class Stream:
    def __init__(self, at):
        self.device = torch.device(at)


def test_a_stream_of_another_device():
    with pytest.raises(binding.PVError, match="stream"):
        operators._Elsewhere(torch.device("cuda", 0), Stream("cuda:1"))
    operators._Elsewhere(torch.device("cuda", 1), None)
