"""What the Python calls on rows of logits refuse before they look at the device: no GPU."""
import pytest
import torch

from paper_2503_23367_b200 import binding as fv


def test_a_place_for_a_gradient_that_is_not_asked_for():
    """Without want_grad nothing would be written there."""
    x = torch.zeros(4, 100)
    t_ids, t_logits = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3)
    for out in (torch.empty_like(x), x):
        with pytest.raises(AssertionError, match="want_grad"):
            fv.fv_distill_topk(x, t_ids, t_logits, out=out)
