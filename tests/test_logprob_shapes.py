"""The shapes that the binding takes result buffers of logits rows in; no GPU."""
import pytest
import torch

from paper_2609_31395_b200 import binding as B


def test_widths_come_from_the_buffer_not_from_its_size():
    assert B._result_rows(torch.zeros(16, 20), 8, None, "top_index") == 20
    assert B._result_rows(torch.zeros(16, 20), 16, 20, "top_logprob") == 20
    assert B._result_rows(torch.zeros(4, 0), 4, None, "top_index") == 0
    assert B._result_rows(torch.zeros(4), 4, 1, "logprob") == 1


@pytest.mark.parametrize("t,n,width", [(None, 1, None), (torch.zeros(20), 4, None), (torch.zeros(3, 5), 4, None), (torch.zeros(4, 5), 4, 6),
                                       (torch.zeros(1, 4, 5), 1, None)])
def test_other_shapes_are_refused(t, n, width):
    with pytest.raises(ValueError):
        B._result_rows(t, n, width, "top_index")
