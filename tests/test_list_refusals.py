"""A teacher's list that the distillation's Python calls refuse before the library is called, so without a GPU."""
import pytest
import torch

from paper_2011_06495_amd import binding as B


def test_logits_without_coordinates():
    """They would be left out of the loss without a word."""
    z, top, label = torch.zeros((3, 20)), torch.zeros((3, 4)), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="no idx"):
        B.mv_distill_loss(z, None, top, label, 2.0, 0.5, 0.5, torch.zeros(3))
    with pytest.raises(ValueError, match="no idx"):
        B.mv_distill_grad(z, None, top, label, 2.0, 0.5, 0.5, torch.zeros((3, 3)), torch.zeros((3, 20)))


def test_coordinates_without_logits():
    z, idx = torch.zeros((3, 20)), torch.zeros((3, 4), dtype=torch.int32)
    with pytest.raises(ValueError, match="no logits"):
        B.mv_distill_loss(z, idx, None, None, 2.0, 0.5, 0.5, torch.zeros(3))
