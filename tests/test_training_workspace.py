"""Workspace sizes of the training step's operators: room for partial results only where
there are some."""
import pytest

import paper_2602_04870_amd as m


@pytest.mark.parametrize("T,Nh,dh,Ne", [(1, 1, 64, 1), (128, 64, 128, 1024), (250, 3, 64, 40),
                                        (4000, 1024, 128, 1024)])
def test_gradient_at_once_needs_no_partial_results(T, Nh, dh, Ne):
    """dW of one chunk of tokens is written at once: what is left are the weights, as of no
    tokens."""
    size = m.mhlmoe_balance_loss_backward_workspace
    assert size(T, Nh, dh, Ne) == size(0, Nh, dh, Ne)


def test_gradient_in_parts_has_room_for_them():
    size = m.mhlmoe_balance_loss_backward_workspace
    one = 4 * 2 * 32 * 128  # a partial result of 2 heads, up to 32 experts
    assert size(500, 3, 64, 40) - size(0, 3, 64, 40) == 2 * 4 * 3 * 64 * 64  # two chunks of 256 tokens
    assert size(1 << 16, 2, 128, 20) - size(0, 2, 128, 20) >= 2 * one
