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


@pytest.mark.parametrize("vocab,most", [(64, 1 << 23), (100, 1 << 23), (1 << 20, 1 << 15)])
def test_a_piece_that_one_launch_takes(lib, vocab, most):
    """A launch has fewer than 2^32 threads: 256 for a token of the piece, 256 for each tile of logits (here: at least 64 x 64)."""
    def size(piece):
        return lib.psgd_head_workspace_bytes(C.byref(head(tokens=(1 << 26) - 3, d=8, vocab=vocab, piece_tokens=piece)), 0)

    assert size(1 << 26) == size(most) != size(most // 2)
    assert size(0) <= size(most)
