"""How a list of gradients is dealt to launches, from the partial sums that it asks a workspace for."""
import pytest

from paper_2606_19025_amd import binding as B

CHUNK = 16384  # values of a chunk of a long list


def partials(*sizes):
    p = 1 << 12  # (an address that is never read)
    grads = (B.moe_grad * len(sizes))(*[B.moe_grad(p, p, n, B.MOE_BF16) for n in sizes])
    return B.moe_grad_norm_workspace_size(grads, len(sizes)) // 8


@pytest.mark.parametrize("past", [1, 100, 2047, 1 << 20])
def test_a_blocks_counter_stays_in_31_bits(past):
    """A block steps from chunk to chunk by the launch's blocks and ends past the last chunk: a launch with fewer
    than a step less than 2^31 chunks would count past an int.  (One gradient of the card's memory may be
    listed that often.)"""
    one = partials((1 << 44) - 1)  # 2^30 chunks: all blocks of one launch
    assert one >= 256
    assert partials((1 << 44) - 1, ((1 << 30) - past) * CHUNK) == 2 * one
    # and what one launch takes: up to 2^30 chunks together
    assert partials(((1 << 30) - past) * CHUNK, past * CHUNK) == one
    assert partials(((1 << 30) - past) * CHUNK, past * CHUNK + 1) == one + min(one, past + 1)
