"""The gated unit and output head of the demonstration: its gradients against automatic differentiation in 64 bits, and that it learns."""
import pytest
import torch

from paper_2509_11254_amd import demo_head

pytestmark = pytest.mark.gpu


def test_gradients_against_autograd():
    model = demo_head.Model(tokens=200, d=72, hidden=136, vocab=333, seed=3)
    tokens, labels = model.batch()
    got = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in model.shapes]
    loss = model.gradients(tokens, labels, got)
    w = [x.bfloat16().double().cpu().requires_grad_() for x in model.weights]
    x = model.table[tokens].double().cpu()
    gate, up = x @ w[0].T, x @ w[1].T
    y = x + (torch.nn.functional.silu(gate) * up) @ w[2].T
    want = torch.nn.functional.cross_entropy(y @ w[3].T, labels.cpu(), ignore_index=-100, reduction="none")
    # activations are rounded to bf16 (2^-9 on average each), some of them to 8 bits with a common scale (a 127th of the largest of 32, so
    # about 2^-8 of a typical element's square mean): a few such errors, none of which adds up
    assert (loss.double().cpu() - want).abs().max() < 0.15
    (want.sum() / (labels >= 0).sum().item()).backward()
    for name, a, b in zip(demo_head.NAMES, got, w):
        error = (a.double().cpu() - b.grad).norm() / b.grad.norm()
        assert error < 0.03, (name, float(error))


def test_it_learns():
    losses = demo_head.run(steps=200)
    first, last = sum(losses[:5]) / 5, sum(losses[-5:]) / 5
    print("loss %.3f -> %.3f" % (first, last))
    # the language's own entropy: the successor with 8/9 of the counted labels, the rest spread over 1000 tokens: about 1.1
    assert 6.5 < first < 9.0
    assert last < 0.6 * first
