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


@pytest.mark.parametrize("dtype,cols", [(psgd.PSGD_BF16, 32 * 2048), (psgd.PSGD_F32, 32 * 1024)])
def test_more_than_one_launch_of_activations(lib, dtype, cols):
    """2^33 pieces of 16 bytes, two to a thread, would be 2^32 threads: refused as sizes, not by the launch."""
    P, rows = 4096, 1 << 20
    for n in (rows, rows + 1):
        assert lib.psgd_act_store(None, n, cols, P, dtype, cols, P, cols, P) == psgd.PSGD_E_SHAPE
        assert lib.psgd_act_restore(None, n, cols, P, cols, P, P, dtype, cols) == psgd.PSGD_E_SHAPE
        assert lib.psgd_act_glu(None, n, cols, 0, dtype, P, None, cols, P, cols, P, P, None, None, cols) == psgd.PSGD_E_SHAPE
        assert lib.psgd_act_glu_backward(None, n, cols, 0, dtype, P, P, None, None, cols, P, cols, P, None, cols) == psgd.PSGD_E_SHAPE
    # (that one row less is taken shows where nothing is launched)
    assert lib.psgd_act_wgrad_workspace_bytes(rows, 8, 32 * 2048, psgd.PSGD_BF16) == 0
    assert lib.psgd_act_wgrad_workspace_bytes(rows - 1, 8, 32 * 2048, psgd.PSGD_BF16) > 0


def test_head_refuses_results_over_inputs(lib):
    """100 tokens, d = 64, 1000 words, bf16 with dW in fp32: X and dX have 12800 bytes, W 128000, dW 256000, labels 800, losses and weights 400."""
    place = dict(x=1 << 20, w=2 << 20, labels=3 << 20, weight=4 << 20, loss=5 << 20, dx=6 << 20, dw=7 << 20)

    def call(desc=None, **change):
        a = dict(place, **change)
        return lib.psgd_head_loss_grad(C.byref(desc or head()), 4096, None, a["x"], a["w"], a["labels"], a["weight"], a["loss"], a["dx"], a["dw"], 0)

    last = dict(x=12800, w=128000, labels=800, weight=400, loss=400, dx=12800, dw=256000)
    for out in ("loss", "dx", "dw"):
        for other in set(place) - {out}:
            # begins in the other's last 16 bytes, or ends in its first
            for at in (place[other] + last[other] // 16 * 16 - 16, place[other] - last[out] // 16 * 16 + 16):
                assert call(**{out: at}) == psgd.PSGD_E_INVALID_ARG, (out, other)
    assert call(dx=place["x"], desc=head(ldx=72)) == psgd.PSGD_E_INVALID_ARG         # X's place, but other rows
    # columns of one buffer: the last of one are the first of the other's
    for shift in (-56, 56, 128 - 56, 56 - 128):
        assert call(dx=place["x"] + 2 * shift, desc=head(ldx=128, lddx=128)) == psgd.PSGD_E_INVALID_ARG, shift
    loss = lib.psgd_head_loss(C.byref(head()), 4096, None, place["x"], place["w"], place["labels"], place["labels"] + 796)
    assert loss == psgd.PSGD_E_INVALID_ARG
