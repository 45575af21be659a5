"""The training operators at the ends of what their arguments may be."""
import pytest
import torch

from paper_2509_11254_amd import psgd

pytestmark = pytest.mark.gpu


def test_losses_of_more_tokens_than_one_launch_takes():
    """More than 2^24 tokens and a small vocabulary: pieces that a launch of 256 threads for each token still takes."""
    tokens, d, vocab = (1 << 24) + 77, 8, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    w = torch.randn((vocab, d), generator=gen, device="cuda").bfloat16()
    x = torch.randn((tokens, d), generator=gen, device="cuda").bfloat16()
    labels = torch.randint(-8, vocab, (tokens,), generator=gen, device="cuda")
    loss = torch.full((tokens,), float("nan"), device="cuda")
    psgd.HeadLoss(tokens, d, vocab, grad=False).loss(x, w, labels, loss)
    for first in range(0, tokens, 1 << 22):
        part = slice(first, min(tokens, first + (1 << 22)))
        logits = x[part].float() @ w.float().t()
        want = torch.logsumexp(logits, 1) - logits.gather(1, labels[part].clamp(min=0)[:, None])[:, 0]
        # eight products summed in fp32, here and there: 8 x 2^-24 of |x| |w|, up to 30, twice in a loss
        assert (loss[part] - torch.where(labels[part] >= 0, want, 0.0)).abs().max() < 1e-4
