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


def test_a_status_that_is_no_int32_word_on_the_device():
    """The kernels write 4 bytes there, on their own device."""
    good = torch.zeros(1, dtype=torch.int32)
    assert fv._word(None, 0) is None and fv._word(12345, 0) == 12345 and fv._word(good, -1) == good.data_ptr()
    for bad, dev in ((good, 0), (torch.zeros(1, dtype=torch.uint8), -1), (torch.zeros(1), -1), (good[:0], -1)):
        with pytest.raises(AssertionError, match="status"):
            fv._word(bad, dev)


def test_every_call_on_rows_of_logits_checks_its_status():
    import inspect
    for call in (fv.fv_token_logprobs, fv.fv_token_logprobs_grad, fv.fv_distill_topk, fv.fv_distill_topk_grad, fv.fv_linear_logprobs):
        assert "_word(status, dev)" in inspect.getsource(call)
