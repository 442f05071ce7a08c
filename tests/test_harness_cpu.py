"""The checks of the tensors that a learner's calls take."""
import pytest
import torch

from paper_1904_04956_amd.harness import checked

CPU = torch.device("cpu")


def test_a_tensor_of_the_right_kind_is_returned():
    t = torch.zeros(3, 4, 5)
    assert checked("t", t, torch.float32, (3, 4, 5), CPU) is t
    assert checked("t", t, torch.float32, torch.Size([3, 4, 5]), CPU) is t


@pytest.mark.parametrize("tensor,error", [
    (None, TypeError), ([0.0] * 4, TypeError), (torch.zeros(3, 4).numpy(), TypeError), (torch.zeros(3, 4, dtype=torch.float64), TypeError),
    (torch.zeros(3, 4, dtype=torch.int64), TypeError), (torch.zeros(4, 3), ValueError), (torch.zeros(4, 3).t(), ValueError), (torch.zeros(3, 4, 1), ValueError),
    (torch.zeros(12), ValueError), (torch.zeros(3, 8)[:, ::2], ValueError), (torch.zeros(1, 4).expand(3, 4), ValueError), (torch.zeros(3, 4, device="meta"), ValueError)], ids=str)
def test_anything_else_is_refused(tensor, error):
    with pytest.raises(error, match="advantage must be"):
        checked("advantage", tensor, torch.float32, (3, 4), CPU)
