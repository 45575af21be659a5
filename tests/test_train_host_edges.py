"""Host-side checks of the training operators at the ends of what their arguments may be, without a GPU: nothing is enqueued."""
import ctypes as C

import pytest

from paper_2509_11254_amd import psgd
from test_train_host import head


@pytest.fixture(scope="module")
def lib():
    return psgd.load_library()


@pytest.mark.parametrize("gradients", [0, 1])
@pytest.mark.parametrize("tokens", [0, 1, 8, 1000])
@pytest.mark.parametrize("piece", [1 << 31, (1 << 63) - 9, (1 << 63) - 4, (1 << 63) - 1])
def test_a_piece_longer_than_the_tokens(lib, piece, tokens, gradients):
    """However many tokens a piece may have, there are no more than there are."""
    one = lib.psgd_head_workspace_bytes(C.byref(head(tokens=tokens, piece_tokens=max(1, tokens))), gradients)
    assert 0 < one < 1 << 30
    assert lib.psgd_head_workspace_bytes(C.byref(head(tokens=tokens, piece_tokens=piece)), gradients) == one
