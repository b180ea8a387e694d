"""CPU check: a workspace at an address that the kernels' words cannot have is refused on the host.  No kernel runs here."""
import ctypes

import pytest
from test_more_operators_abi import balance, block_norm_backward, product


@pytest.mark.parametrize("call", [balance, block_norm_backward, product])
@pytest.mark.parametrize("at", [1, 2, 3, 4, 6, 7])
def test_words_at_odd_addresses(call, at):
    assert call(ws=ctypes.c_void_p(0x1000 + at)) == 3
