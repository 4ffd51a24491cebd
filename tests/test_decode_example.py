"""The example of decoding over virtual ranks: whatever the number of ranks, the joined result is the
undivided cache's."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ranks,steps", [(2, 20), (5, 100), (7, 33)])
def test_ranks_join_to_the_undivided_attention(ranks, steps):
    from examples import decode_ranks
    # The ranks' shares are the same 8-bit rows; weights, sums and joins are held to about 2^-17 and 32 bits.
    assert decode_ranks.main(ranks, steps) < 1e-4
